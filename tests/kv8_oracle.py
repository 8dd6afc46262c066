"""Plain forms of the 8-bit cache and of the pages that rows share, in numpy, one block, row or fork at a time, in 64
bits, written from include/wf_kv.h.  Test infrastructure only."""
import numpy as np

LEAST, MOST = -100, 119


def code_values():
    """The value of each of the 256 codes, from its bits."""
    out = np.empty(256)
    for c in range(256):
        e, m = c >> 3 & 15, c & 7
        v = np.nan if c & 0x7f == 0x7f else (8 + m) * 2.0 ** (e - 10) if e else m * 2.0 ** -9
        out[c] = -v if c & 0x80 else v
    return out


VALUES = code_values()
_GRID = VALUES[:0x7f]                       # 0 .. 448, ascending
_HALF = (_GRID[1:] + _GRID[:-1]) / 2        # exact


def codes(x):
    """Nearest codes of 64-bit values already divided by the scale, ties to the even code, above 448 taken as 448."""
    a = np.abs(x)
    i = np.searchsorted(_HALF, a, side="left")              # a in (half[i-1], half[i]]
    tie = (i < len(_HALF)) & (a == _HALF[np.minimum(i, len(_HALF) - 1)])
    i = np.where(tie & (i % 2 == 1), i + 1, i)              # half-way: up where the lower code is odd
    return (i | np.where(np.signbit(x), 0x80, 0)).astype(np.uint8)


def least_power(most):
    """The least e for which `most` does not pass 448 * 2^e."""
    if most == 0:
        return LEAST
    m, x = np.frexp(np.float64(most))                       # most = m 2^x, 1/2 <= m < 1; 448 = 7/8 2^9
    return int(min(max(x - 9 + (m > 0.875), LEAST), MOST))


class Cache8:
    """A cache as bytes [n_blocks, Hk, 2 B D + 16]."""

    def __init__(self, n_blocks, hk, b, d, rng=None):
        self.n, self.hk, self.b, self.d = n_blocks, hk, b, d
        size = (n_blocks, hk, 2 * b * d + 16)
        self.bytes = np.zeros(size, np.uint8) if rng is None else rng.integers(0, 256, size, dtype=np.uint8)

    def keys(self):
        n = self.b * self.d
        return self.bytes[..., :n].reshape(self.n, self.hk, self.b, self.d)

    def value_codes(self):
        """[n, Hk, B, D] (a copy)."""
        n, b, d = self.b * self.d, self.b, self.d
        return self.bytes[..., n:2 * n].reshape(self.n, self.hk, b // 4, d, 4).swapaxes(-1, -2).reshape(self.n, self.hk, b, d)

    def put_values(self, blk, h, code):
        n, b, d = self.b * self.d, self.b, self.d
        self.bytes[blk, h, n:2 * n] = code.reshape(b // 4, 4, d).swapaxes(-1, -2).reshape(-1)

    def scales(self):
        n = 2 * self.b * self.d
        return np.ascontiguousarray(self.bytes[..., n:n + 8]).view(np.float32)

    def put_scale(self, blk, h, i, e):
        n = 2 * self.b * self.d + 4 * i
        self.bytes[blk, h, n:n + 4] = np.array([2.0 ** e], np.float32).view(np.uint8)

    def put_run(self, blk, offs, k, v):
        """fp32 tokens k, v [len(offs), Hk, D] of one block, from one call."""
        for h in range(self.hk):
            bad = ~(np.isfinite(k[:, h]).all(-1) & np.isfinite(v[:, h]).all(-1))
            for i, x in enumerate((k[:, h], v[:, h])):
                held = self.keys()[blk, h].copy() if i == 0 else self.value_codes()[blk, h]
                e = least_power(np.abs(x[~bad]).max() if (~bad).any() else 0)
                if 0 not in offs:
                    old = int(np.log2(self.scales()[blk, h, i]))
                    e = max(e, old)
                    if e != old:
                        nan = (held & 0x7f) == 0x7f
                        held = np.where(nan, held, codes(np.where(nan, 0, VALUES[held]) * 2.0 ** (old - e)))
                with np.errstate(invalid="ignore"):
                    new = codes(np.where(bad[:, None], 0, x).astype(np.float64) / 2.0 ** e)
                new[bad] = 0x7f if i == 0 else 0
                held[list(offs)] = new
                if i == 0:
                    self.bytes[blk, h, :self.b * self.d] = held.reshape(-1)
                else:
                    self.put_values(blk, h, held)
                self.put_scale(blk, h, i, e)

    def put(self, slots, k, v):
        """A call's tokens [T, Hk, D]; slots below 0 or past the cache store nothing."""
        t = 0
        while t < len(slots):
            blk, n = slots[t] // self.b, 1
            if slots[t] < 0 or blk >= self.n:
                t += 1
                continue
            while t + n < len(slots) and slots[t + n] >= 0 and slots[t + n] // self.b == blk:
                n += 1
            self.put_run(int(blk), [int(s % self.b) for s in slots[t:t + n]], k[t:t + n], v[t:t + n])
            t += n

    def get(self, slots):
        """Keys and values [T, Hk, D] in 64 bits."""
        slots = np.asarray(slots)
        blk, off = slots // self.b, slots % self.b
        s = self.scales().astype(np.float64)
        kc = self.keys()[blk, :, off]
        k = VALUES[kc] * s[blk, :, 0][..., None]
        n = self.b * self.d
        vc = self.bytes[..., n:2 * n].reshape(self.n, self.hk, self.b // 4, self.d, 4)[blk, :, off // 4, :, off % 4]
        v = VALUES[vc] * s[blk, :, 1][..., None]
        return k, np.where((kc[..., :1] & 0x7f) == 0x7f, np.nan, v)


def attend(q, cache, table, kv_len, q_off, pos, scale, window):
    """Outputs [T, Hq, D] in 64 bits, sum p |v|, the largest sum of |q k| and the largest probability times value scale of
    each query's head (for error bounds)."""
    q = np.asarray(q, np.float64)
    T, hq, d = q.shape
    g = hq // cache.hk
    out, mag, dots, top = np.zeros_like(q), np.zeros_like(q), np.zeros((T, hq)), np.zeros((T, hq))
    scales = cache.scales().astype(np.float64)
    for r in range(len(kv_len)):
        n, t0, t1 = int(kv_len[r]), int(q_off[r]), int(q_off[r + 1])
        if n == 0 or t0 == t1:
            continue
        j = np.arange(n)
        blocks = table[r, j // cache.b].astype(np.int64)
        k, v = cache.get(blocks * cache.b + j % cache.b)
        p = np.asarray(pos[t0:t1], np.int64)[:, None]
        see = (j[None] <= p) & ((j[None] > p - window) if window else True)
        some = see.any(-1)
        for h in range(hq):
            x, kk, vv = q[t0:t1, h], k[:, h // g], v[:, h // g]
            s = np.where(see, scale * (x @ kk.T), -np.inf)
            w = np.exp(s - np.where(some, s.max(-1), 0)[:, None])
            w = w / np.where(some, w.sum(-1), 1)[:, None]
            out[t0:t1, h], mag[t0:t1, h] = w @ vv, w @ np.abs(vv)
            dots[t0:t1, h] = abs(scale) * np.where(see, np.abs(x) @ np.abs(kk).T, 0).max(-1)
            top[t0:t1, h] = (w * scales[blocks, h // g, 1]).max(-1)
    return out, mag, dots, top


def fork(forks, lens, pool, ring, table, shared, block):
    """One fork (src, dst, tokens) after the other, all of them on the rows as they were."""
    lens0, n, (head, free) = [int(x) for x in lens], len(ring), (int(pool[0]), int(pool[1]))
    lens, table, shared = list(lens0), table.copy(), shared.copy()
    granted, moves, upto, taken = [], [], 0, 0
    for src, dst, want in forks:
        ok = 0 <= src < len(lens0) and 0 <= dst < len(lens0) and src != dst and want >= 0 and lens0[dst] == 0
        old = new = -1
        if ok:
            k = min(want, lens0[src])
            need = int(k % block > 0)
            upto += need
            ok = not need or upto <= free
        if ok:
            for j in range(k // block):
                table[dst, j] = table[src, j]
                shared[table[src, j]] += 1
            if need:
                old, new = table[src, k // block], ring[(head + taken) % n]
                table[dst, k // block] = new
                taken += 1
            lens[dst] = k
        granted.append(int(ok))
        moves.append((old, new))
    return dict(lens=np.array(lens), pool=np.array([(head + taken) % n, free - taken]), shared=shared, granted=np.array(granted),
                moves=np.array(moves).reshape(-1, 2).T, table=table)


def release(ends, lens, pool, ring, table, shared, block):
    """One row's block after the other; then the blocks that nobody holds, by id."""
    left, ring, n = shared.copy(), ring.copy(), len(ring)
    for r, e in enumerate(ends):
        if e:
            for j in range(-(-int(lens[r]) // block)):
                left[table[r, j]] -= 1
    freed = [b for b in range(n) if left[b] < 0]
    for i, b in enumerate(freed):
        ring[(int(pool[0]) + int(pool[1]) + i) % n] = b
        left[b] = 0
    return dict(lens=np.where(np.asarray(ends) != 0, 0, lens), pool=np.array([int(pool[0]), int(pool[1]) + len(freed)]), shared=left, ring=ring)


def compact(keep, lens, pool, ring, table, shared, block):
    n = len(ring)
    free = {int(ring[(int(pool[0]) + i) % n]) for i in range(int(pool[1]))}
    goes = [b for b in range(keep, n) if b not in free]
    holes = [b for b in range(keep) if b in free]
    most = min(keep, n - keep)
    moves = np.full((2, most), -1)
    table = table.copy()
    if len(goes) > len(holes):
        return dict(done=np.array([0]), moves=moves, table=table)
    to = dict(zip(goes, holes))
    moves[0, :len(goes)], moves[1, :len(goes)] = goes, holes[:len(goes)]
    for r in range(len(lens)):
        for j in range(-(-int(lens[r]) // block)):
            table[r, j] = to.get(int(table[r, j]), table[r, j])
    out = np.where([b in free for b in range(keep)], 0, shared[:keep])
    for b, h in to.items():
        out[h] = shared[b]
    left = holes[len(goes):]
    return dict(done=np.array([1]), moves=moves, table=table, shared=out, pool=np.array([0, len(left)]),
                ring=np.array(left + [-1] * (keep - len(left))))
