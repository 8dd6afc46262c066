"""Plain forms of the paged-cache operators in numpy, one row, token or head at
a time, in 64 bits, written from include/wf_kv.h.  Test infrastructure only."""
import numpy as np

GRID = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])


def bf16(x):
    """Nearest bf16 (ties to even) of fp32 values, as fp32 and as bits."""
    u = np.asarray(x, np.float32).view(np.uint32).astype(np.uint64)
    bits = ((u + 0x7fff + ((u >> 16) & 1)) >> 16).astype(np.uint16)
    bits = np.where(np.isnan(x), np.uint16(0x7fc0), bits)
    return (bits.astype(np.uint32) << 16).view(np.float32), bits


def step(new, lens, pool, ring, table, block, n_tokens):
    """One row after the other."""
    new, lens = [int(x) for x in new], [int(x) for x in lens]
    ring, table = ring.copy(), table.copy()
    n, width, (head, free) = len(ring), table.shape[1], (int(pool[0]), int(pool[1]))
    left, upto, back = free, 0, 0
    len_out, granted, q_off, slot, pos, taken = [], [], [0], [], [], 0
    gives = []
    for r, (f, have) in enumerate(zip(new, lens)):
        blocks = -(-have // block)
        grow = max(f, 0)
        if f < 0:
            gives += [int(b) for b in table[r, :blocks]]
            granted.append(0)
            len_out.append(0)
        else:
            want = -(-(have + grow) // block)
            fits = have + grow <= width * block
            need = want - blocks if fits else 0
            upto += need
            ok = fits and (need == 0 or upto <= free)
            if ok:
                for i in range(need):
                    table[r, blocks + i] = ring[(head + taken + i) % n]
                taken += need
            granted.append(int(ok))
            len_out.append(have + grow if ok else have)
        q_off.append(q_off[-1] + grow)
        for i in range(grow):
            p = have + i
            pos.append(p)
            slot.append(int(table[r, p // block]) * block + p % block if granted[-1] else -1)
    for i, b in enumerate(gives):
        ring[(head + free + i) % n] = b
    pad = n_tokens - len(pos)
    if pad > 0:
        pos, slot = pos + [0] * pad, slot + [-1] * pad
    return dict(lens=np.array(len_out), pool=np.array([(head + taken) % n, free - taken + len(gives)]),
                q_off=np.array(q_off), slot=np.array(slot[:n_tokens], np.int64), pos=np.array(pos[:n_tokens]),
                granted=np.array(granted), ring=ring, table=table)


def normed_rotated(x, weight, eps, cos_sin, pos, rot, interleaved):
    """x [T, H, D] in 64 bits."""
    x = np.asarray(x, np.float64)
    if weight is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * np.asarray(weight, np.float64)
    if not rot:
        return x
    h = rot // 2
    c = cos_sin.astype(np.float64)[pos][:, None, :h]
    s = cos_sin.astype(np.float64)[pos][:, None, h:]
    y = x.copy()
    i, j = (np.arange(0, rot, 2), np.arange(1, rot, 2)) if interleaved else (np.arange(h), np.arange(h, rot))
    y[..., i] = x[..., i] * c - x[..., j] * s
    y[..., j] = x[..., j] * c + x[..., i] * s
    return y


def quantised(x):
    """Codes and scale bits of fp32 vectors [.., D]: the definition, exactly
    (all comparisons of fp32 values, as 64-bit ones)."""
    x = np.asarray(x, np.float32)
    most = np.abs(x).max(-1)
    s, bits = bf16(most * np.float32(1 / 6))
    ok = np.isfinite(x).all(-1)
    s, bits = np.where(ok, s, np.float32(np.nan)), np.where(ok, bits, np.uint16(0x7fc0))
    with np.errstate(invalid="ignore"):
        return quantised_with(x.astype(np.float64), s), bits


def quantised_with(x, s):
    """Codes of 64-bit vectors under given scales."""
    a, f = np.abs(x), np.asarray(s, np.float64)[..., None]
    code = sum(((a > t * f) if k % 2 == 0 else (a >= t * f)).astype(np.uint8)
               for k, t in enumerate((0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0)))
    return code | (x < 0).astype(np.uint8) << 3


def values(code):
    return GRID[code & 7] * np.where(code & 8, -1.0, 1.0)


class Cache:
    """A cache as bytes [n_blocks, Hk, B * (D + 4)]."""

    def __init__(self, n_blocks, hk, b, d, rng=None):
        self.n, self.hk, self.b, self.d = n_blocks, hk, b, d
        size = (n_blocks, hk, b * (d + 4))
        self.bytes = np.zeros(size, np.uint8) if rng is None else rng.integers(0, 256, size, dtype=np.uint8)

    def parts(self):
        b, d = self.b, self.d
        n = b * d // 2
        c = self.bytes
        return (c[..., :n].reshape(self.n, self.hk, b, d // 2), c[..., n:2 * n].reshape(self.n, self.hk, d // 2, b),
                np.ascontiguousarray(c[..., 2 * n:]).view(np.uint16).reshape(self.n, self.hk, 2, b))

    def put(self, slot, k, v):
        """fp32 vectors [Hk, D] at a slot."""
        b, d = self.b, self.d
        blk, off = divmod(int(slot), b)
        n = b * d // 2
        for h in range(self.hk):
            cell = self.bytes[blk, h]
            code, bits = quantised(k[h])
            cell[off * d // 2:(off + 1) * d // 2] = code[0::2] | code[1::2] << 4
            cell[2 * n:].view(np.uint16)[off] = bits
            code, bits = quantised(v[h])
            cell[n:2 * n].reshape(d // 2, b)[:, off] = code[:d // 2] | code[d // 2:] << 4
            cell[2 * n:].view(np.uint16)[b + off] = bits

    def get(self, slots):
        """Keys and values [T, Hk, D] in 64 bits."""
        kc, vc, sc = self.parts()
        slots = np.asarray(slots)
        blk, off = slots // self.b, slots % self.b
        s = (sc.astype(np.uint32) << 16).view(np.float32).astype(np.float64)
        c = kc[blk, :, off]
        k = values(np.stack([c & 15, c >> 4], -1).reshape(*c.shape[:-1], self.d)) * s[blk, :, 0, off][..., None]
        c = vc[blk, :, :, off]
        v = values(np.concatenate([c & 15, c >> 4], -1)) * s[blk, :, 1, off][..., None]
        return k, v


def attend(q, cache, table, kv_len, q_off, pos, scale, window):
    """Outputs [T, Hq, D] in 64 bits, sum p |v| and the largest sum of |q k| of
    each query (for error bounds)."""
    q = np.asarray(q, np.float64)
    T, hq, d = q.shape
    g = hq // cache.hk
    out, mag, dots = np.zeros_like(q), np.zeros_like(q), np.zeros((T, hq))
    for r in range(len(kv_len)):
        n = int(kv_len[r])
        if n == 0:
            continue
        j = np.arange(n)
        k, v = cache.get(table[r, j // cache.b].astype(np.int64) * cache.b + j % cache.b)
        for t in range(int(q_off[r]), int(q_off[r + 1])):
            see = j <= pos[t]
            if window:
                see &= j > pos[t] - window
            if not see.any():
                continue
            for h in range(hq):
                kk, vv = k[see, h // g], v[see, h // g]
                s = scale * (kk @ q[t, h])
                p = np.exp(s - s.max())
                p /= p.sum()
                out[t, h], mag[t, h] = p @ vv, p @ np.abs(vv)
                dots[t, h] = abs(scale) * (np.abs(kk) @ np.abs(q[t, h])).max()
    return out, mag, dots
