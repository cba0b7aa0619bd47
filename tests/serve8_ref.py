"""Plain implementations of the cache held in 8 bits as sagebwd_serve.h defines it; they share nothing with the library."""
import numpy as np

F = np.float32


class Block:
    """What a block of tokens of a head holds of K (or of V): codes [block, d], the largest magnitude, and how many tokens are held."""

    def __init__(self, block, d):
        self.codes, self.a, self.held = np.zeros((block, d), np.int64), F(0), 0

    def store(self, o, x):
        """Tokens o .. of the block, float32 [n, d] (means taken off)."""
        with np.errstate(all="ignore"):
            m = F(np.abs(x).max())                     # (numpy's max hands a NaN on)
            a = F(np.maximum(m, self.a)) if o > 0 else m
            if not a < F(2.0 ** 127):
                a = F(np.nan)
            elif a < F(2.0 ** -100):
                a = F(0)
            if o > 0 and a > self.a:
                f = F(self.a / a)
                self.codes[:o] = np.rint(self.codes[:o].astype(F) * f).astype(np.int64)
            r = F(F(127) / a) if a > 0 else F(0)
            new = np.rint(x.astype(F) * r) if a > 0 else np.zeros_like(x)
        self.codes[o:o + len(x)] = new.astype(np.int64)
        self.a, self.held = a, o + len(x)

    def values(self):
        """float64 [held, d]"""
        with np.errstate(all="ignore"):
            return self.codes[:self.held] * (np.float64(self.a) / 127)

    def read(self):
        """float32 [held, d], before the rounding to bf16"""
        with np.errstate(all="ignore"):
            return self.codes[:self.held].astype(F) * F(self.a / F(127))


class Pages:
    """Tokens of any slots of a cache, stored call by call."""

    def __init__(self, H, d, page, block):
        self.H, self.d, self.page, self.block, self.blocks = H, d, page, block, {}

    def append(self, K, V, slots):
        """float32 [T, H, d] (means taken off); slots as a list, tokens of a block one after the other."""
        begin = 0
        for i in range(1, len(slots) + 1):
            if i == len(slots) or slots[i] != slots[i - 1] + 1 or slots[i] % self.block == 0:
                if slots[begin] >= 0:
                    for h in range(self.H):
                        for which, x in ((0, K), (1, V)):
                            key = (slots[begin] // self.block, h, which)
                            self.blocks.setdefault(key, Block(self.block, self.d)).store(slots[begin] % self.block, np.asarray(x[begin:i, h], F))
                begin = i

    def gather(self, slots, which, how="values"):
        """[T, H, d] of stored slots"""
        out = np.zeros((len(slots), self.H, self.d), np.float64 if how == "values" else F)
        cache = {}
        for t, s in enumerate(slots):
            for h in range(self.H):
                key = (s // self.block, h, which)
                if key not in cache:
                    cache[key] = getattr(self.blocks[key], how)()
                out[t, h] = cache[key][s % self.block]
        return out


def places(d, page):
    """Bytes of K's and V's codes, int [page, d] each, and of the pair of magnitudes, [page], in a head's part of a page."""
    t, c = np.arange(page)[:, None], np.arange(d)[None]
    b, o = t // 32, t % 32 // 8
    k = 32 * d * b + 2048 * (c // 64) + 1024 * (t % 8 // 4) + 256 * (c % 64 // 16) + 64 * o + 16 * (t % 4) + c % 16
    v = page * d + 32 * d * b + 1024 * (c // 32) + 256 * o + 16 * (c % 16) + 8 * (c % 32 // 16) + t % 8
    return k, v, 2 * page * d + 8 * (np.arange(page) // 32)


def decode(part, d, page):
    """(K's codes, V's codes [page, d], a_K, a_V [page]) of one head's part of a page (uint8 bytes)."""
    part = np.ascontiguousarray(part, np.uint8)
    assert part.size == 2 * page * d + max(16, page // 4)
    k, v, a = places(d, page)
    floats = part[2 * page * d:2 * page * d + page // 4].view(F).reshape(-1, 2)
    at = (a - 2 * page * d) // 8
    return part[k].view(np.int8), part[v].view(np.int8), floats[at, 0], floats[at, 1]
