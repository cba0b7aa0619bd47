"""Plain implementations, in 64 bits and token by token, of what sagebwd_serve.h defines; they share nothing with the library."""
import math

import numpy as np


def bf16_round(x):
    """float32 array -> nearest bf16 number (ties to even), as float32."""
    u = np.asarray(x, np.float32).view(np.uint32).astype(np.uint64)
    u = (u + 0x7FFF + ((u >> 16) & 1)) & 0xFFFF0000
    return u.astype(np.uint32).view(np.float32)


def quantise(x, group):
    """(codes -7 .. 7, scales, values) of float32 [..., d], the decisions in FP32 as the header has them."""
    x = np.asarray(x, np.float32)
    g = x.reshape(x.shape[:-1] + (x.shape[-1] // group, group))
    with np.errstate(all="ignore"):
        a = np.abs(g).max(-1)                          # (numpy's max hands a NaN on)
        s = a / np.float32(7)
        s = ((s.view(np.uint32).astype(np.uint64) + 0x7FFFF) & 0xFFF80000).astype(np.uint32).view(np.float32)
        code = np.rint(g / s[..., None])
    tiny, bad = a < np.float32(2.0 ** -100), ~(a < np.float32(2.0 ** 127))
    code = np.where((tiny | bad)[..., None], 0, code)
    s = np.where(tiny, np.float32(0), np.where(bad, np.float32(np.nan), s))
    value = (code * s[..., None]).astype(np.float32).reshape(x.shape)
    return code.astype(np.int64).reshape(x.shape), s, value


def decode_page(part, d, page, group):
    """(K, V) float32 [page, d] of one head's part of a page (uint8 bytes), by the header's formulas."""
    part = np.asarray(part, np.uint8)
    assert part.size == page * (d + 4 * d // group)
    word = lambda at, n: int.from_bytes(part[at:at + n].tobytes(), "little")  # noqa: E731
    bf = lambda at: np.uint32(word(at, 2) << 16).reshape(1).view(np.float32)[0]  # noqa: E731
    K, V = np.zeros((page, d), np.float32), np.zeros((page, d), np.float32)
    ks, vs = page * d, page * d + page * d // group * 2
    with np.errstate(all="ignore"):        # (bytes that nothing was stored in may be any scale)
        _decode(K, V, word, bf, ks, vs, d, page, group)
    return K, V


def _decode(K, V, word, bf, ks, vs, d, page, group):
    for t in range(page):
        o, i = divmod(t, 8)
        for c in range(d):
            j, p, r = c // 32, c % 32 // 8, c % 8
            s = (o * d // group + c // group) * 16 + 2 * i
            n = word(t * d // 2 + p * d // 8 + 4 * j, 4) >> 4 * (r // 2 + 4 * (r % 2)) & 15
            K[t, c] = np.float32(n - 8) * bf(ks + s)
            h, j, m = c // 64, c % 64 // 16, c % 16
            n = word(page * d // 2 + o * 4 * d + 256 * h + 16 * m + 2 * i, 2) >> 4 * j & 15
            V[t, c] = np.float32(n - 8) * bf(vs + s)


def plan(held, added, table, stack, count, page, rows):
    """The dictionary of a plan's outputs; `table` (a list of lists) is changed."""
    slots, positions, cu, lengths, granted = [], [], [0], [], []
    columns = len(table[0]) if table else 1
    tokens, needs, left = 0, 0, count
    for r, (a, n) in enumerate(zip(held, added)):
        valid = a >= 0 and n >= 0 and a + n <= columns * page
        n = n if valid else 0
        need = math.ceil((a + n) / page) - math.ceil(a / page) if valid else 0
        tokens, needs = tokens + n, needs + need
        ok = valid and tokens <= rows and (need == 0 or needs <= count)
        for k in range(need if ok else 0):
            left -= 1
            table[r][math.ceil(a / page) + k] = stack[left]
        for t in range(a, a + n):
            slots.append(table[r][t // page] * page + t % page if ok else -1)
            positions.append(t if ok else 0)
        cu.append(min(tokens, rows))
        lengths.append(a + n if ok else a)
        granted.append(int(ok))
    pad = max(0, rows - len(slots))
    return dict(slots=(slots + [-1] * pad)[:rows], positions=(positions + [0] * pad)[:rows], cu_new=cu, lengths=lengths, granted=granted,
                free_left=[left])


def attention(q, k, v, n_new, causal, scale, v_mean=None):
    """One request: q [n, Hq, d], k, v [L, H, d] (float64) -> O [n, Hq, d], LSE [Hq, n], A [n, Hq, d] = sum p |v| / sum p."""
    n, Hq, d = q.shape
    L, H = k.shape[0], k.shape[1]
    O, A, lse = np.zeros((n, Hq, d)), np.zeros((n, Hq, d)), np.full((Hq, n), -np.inf)
    for h in range(Hq):
        kh, vh = k[:, h // (Hq // H)], v[:, h // (Hq // H)]
        for i in range(n):
            sees = min(L, L - n + i + 1) if causal else L
            if sees <= 0:
                continue
            z = (kh[:sees] @ q[i, h]) * scale
            top = z.max()
            p = np.exp(z - top)
            O[i, h] = p @ vh[:sees] / p.sum() + (0 if v_mean is None else v_mean[h // (Hq // H)])
            A[i, h] = p @ np.abs(vh[:sees]) / p.sum()
            lse[h, i] = top + np.log(p.sum())
    return O, lse, A


def rotary(x, positions, inv_freq, sections, adjacent, inverse=False):
    """x [T, H, d], positions [axes, T] -> turned, float64."""
    x = np.asarray(x, np.float64)
    y, half = x.copy(), len(inv_freq)
    axis = np.repeat(np.arange(len(sections)), sections)
    angle = np.asarray(positions, np.float64)[axis].T * np.asarray(inv_freq, np.float64)      # [T, half]
    c, s = np.cos(angle)[:, None], np.sin(angle)[:, None] * (-1 if inverse else 1)
    one = np.arange(half) * (2 if adjacent else 1)
    two = one + (1 if adjacent else half)
    y[..., one], y[..., two] = x[..., one] * c - x[..., two] * s, x[..., two] * c + x[..., one] * s
    return y
