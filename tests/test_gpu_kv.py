"""The paged 4-bit cache on the GPU against the 64-bit oracle of kv_oracle.py:
block tables and slots, norm + rotation + store, load, attention."""
import numpy as np
import pytest
import torch

import kv_oracle as K
import paper_2609_03335_amd as pkg

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
UNIT = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11}      # of rounding to nearest


@pytest.fixture(scope="module", autouse=True)
def gpu():
    assert torch.cuda.is_available(), "GPU tests need a HIP device"


def ctx_of(hq=8, hk=2, d=64, b=16, n=64, width=8, dtype="bf16"):
    return pkg.KVContext(0, q_heads=hq, kv_heads=hk, head_dim=d, block_tokens=b, n_blocks=n, max_blocks=width, dtype=dtype)


def dev(x, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(x)).to(DEV)
    return t if dtype is None else t.to(dtype)


# ---- block tables and slots --------------------------------------------------------------------

def random_step(rng, rows, b, width, spare, released=0.2, most_new=60):
    lens = rng.integers(0, width * b + 1, rows) * (rng.random(rows) < 0.8)
    new = np.where(rng.random(rows) < 0.5, 1, rng.integers(0, most_new, rows))
    new = np.where(rng.random(rows) < released, -1, new)
    have = -(-lens // b)
    need = np.where((new >= 0) & (lens + new <= width * b), -(-(lens + np.maximum(new, 0)) // b) - have, 0)
    free = max(0, int(need.sum() * spare))
    n = max(1, int(have.sum()) + free)
    ids = rng.permutation(n).astype(np.int32)
    table = np.full((rows, width), -1, np.int32)
    at = 0
    for r in range(rows):
        table[r, :have[r]] = ids[at:at + have[r]]
        at += have[r]
    head = int(rng.integers(0, n))
    ring = np.full(n, -7, np.int32)
    ring[(head + np.arange(free)) % n] = ids[at:at + free]
    return lens.astype(np.int32), new.astype(np.int32), table, ring, np.array([head, free], np.int32)


def check_step(lens, new, table, ring, pool, b, pad=0, cut=0):
    tokens = max(0, int(np.maximum(new, 0).sum()) + pad - cut)
    want = K.step(new, lens, pool, ring, table, b, tokens)
    with ctx_of(b=b, n=len(ring), width=table.shape[1]) as ctx:
        t, r = dev(table), dev(ring)
        args = (ctx, dev(new), tokens, dev(lens), dev(pool), r, t)
        for _ in range(2):   # the inputs are left as they were: a second call gives the same
            got = pkg.kv_step(*args)
        got = dict(zip(("lens", "pool", "q_off", "slot", "pos", "granted"), got), ring=r, table=t)
        for name, x in want.items():
            assert np.array_equal(got[name].cpu().numpy(), x), name


@pytest.mark.parametrize("b", [16, 32, 256])
@pytest.mark.parametrize("rows", [1, 2, 63, 64, 65, 1023, 1024, 1025, 2500, 4096, 4097, 9000])
def test_step(rows, b):
    rng = np.random.default_rng(rows * 1000 + b)
    for spare in (1.0, 0.5):
        check_step(*random_step(rng, rows, b, 6, spare), b, pad=5)


def test_step_edges():
    rng = np.random.default_rng(0)
    z = np.zeros(0, np.int32)
    # no rows; no tokens; every row released; none free; more tokens than asked for, and fewer
    check_step(z, z, np.zeros((0, 4), np.int32), np.arange(9, dtype=np.int32), np.array([3, 6], np.int32), 16, pad=3)
    check_step(*random_step(rng, 40, 16, 5, 1.0, most_new=1), 16)
    check_step(*random_step(rng, 40, 16, 5, 1.0, released=1.0), 16)
    check_step(*random_step(rng, 40, 16, 5, 0.0), 16)
    check_step(*random_step(rng, 40, 16, 5, 1.0), 16, pad=1000)
    check_step(*random_step(rng, 40, 16, 5, 1.0), 16, cut=37)


def test_step_one_long_prompt():
    # thousands of blocks for one row, and as many released by another
    b, width = 16, 8000
    lens, new = np.array([0, 100000, 5], np.int32), np.array([120000, -1, 1], np.int32)
    n = 7500 + 6250 + 1
    ids = np.random.default_rng(3).permutation(n).astype(np.int32)
    table = np.full((3, width), -1, np.int32)
    table[1, :6250], table[2, 0] = ids[:6250], ids[6250]
    ring = np.full(n, -1, np.int32)
    ring[(n - 10 + np.arange(7500)) % n] = ids[6251:]
    check_step(lens, new, table, ring, np.array([n - 10, 7500], np.int32), b)


@pytest.mark.parametrize("rows", [40, 5000])
def test_step_sums_past_32_bits(rows):
    """Rows that ask for far more than fits: offsets stop at 2^31 - 1, later rows are placed as if
    they were right; needs beyond 2^32 blocks in all leave nothing for the rows after."""
    b, n = 16, 9
    new = np.ones(rows, np.int32)
    new[:7] = 2 ** 31 - 1
    off = np.minimum(np.concatenate([[0], np.cumsum(new.astype(np.int64))]), 2 ** 31 - 1)
    with ctx_of(b=b, n=n, width=4) as ctx:
        table = torch.full((rows, 4), -1, dtype=torch.int32, device=DEV)
        ring, pool = torch.arange(n, dtype=torch.int32, device=DEV), torch.tensor([0, n], dtype=torch.int32, device=DEV)
        lens, pool, q_off, slot, pos, granted = pkg.kv_step(ctx, dev(new), 300, dev(np.zeros(rows, np.int32)), pool, ring, table)
        assert np.array_equal(q_off.cpu().numpy(), off)
        want = np.zeros(rows, np.int32)
        want[7:7 + n] = 1
        assert np.array_equal(granted.cpu().numpy(), want) and np.array_equal(lens.cpu().numpy(), want)
        assert pool.tolist() == [0, 0] and (slot == -1).all() and np.array_equal(pos.cpu().numpy(), np.arange(300))
        assert table[7:7 + n, 0].tolist() == list(range(n)) and (table[7:7 + n, 1:] == -1).all()
    width, rows = 1 << 22, 1100 if rows == 40 else 4200
    with ctx_of(b=b, n=n, width=width) as ctx:
        new = dev(np.full(rows, width * b, np.int32))
        new[-1] = 1
        table = torch.empty(rows, width, dtype=torch.int32, device=DEV)
        pool = torch.tensor([0, n], dtype=torch.int32, device=DEV)
        lens, pool, q_off, slot, pos, granted = pkg.kv_step(ctx, new, 10, torch.zeros_like(new), pool, ring, table)
        assert not granted.any() and not lens.any() and pool.tolist() == [0, n] and (slot == -1).all()


def test_step_invalid_device_values_stay_in_bounds():
    """Lengths, counters and ring contents outside their range: unspecified
    results, but nothing outside the arrays is written."""
    rows, b, width, n = 70, 16, 4, 50
    rng = np.random.default_rng(5)
    wild = lambda k: rng.integers(-2 ** 31, 2 ** 31 - 1, k).astype(np.int32)
    with ctx_of(b=b, n=n, width=width) as ctx:
        for pool in ([-5, 10 ** 9], [10 ** 9, -3], [7, 50]):
            guard = torch.full((64 + rows * width + 64,), 77, dtype=torch.int32, device=DEV)
            ring = torch.full((64 + n + 64,), 78, dtype=torch.int32, device=DEV)
            table = guard[64:-64].view(rows, width)
            table.copy_(dev(wild(rows * width)).view(rows, width))
            pkg.kv_step(ctx, dev(wild(rows)), 500, dev(wild(rows)), dev(np.array(pool, np.int32)), ring[64:-64], table)
            torch.cuda.synchronize()
            for g, x in ((guard, 77), (ring, 78)):
                assert (g[:64] == x).all() and (g[-64:] == x).all()


# ---- store and load ----------------------------------------------------------------------------

def store_case(rng, hq, hk, d, b, T, dtype, rot, pad=0, scale=1.0):
    width = (hq + 2 * hk) * d + pad
    qkv = dev((rng.standard_normal((T, width)) * scale).astype(np.float32), TYPES[dtype])
    part = lambda a, n: qkv[:, a * d:(a + n) * d].unflatten(-1, (n, d))
    n = T // b + 3
    slots = rng.permutation(n * b)[:T].astype(np.int64)
    n_pos = 977
    angle = np.arange(n_pos)[:, None] * 1e4 ** (-np.arange(0, max(rot, 2), 2) / max(rot, 2))
    cs = np.concatenate([np.cos(angle), np.sin(angle)], 1).astype(np.float32)
    return part(0, hq), part(hq, hk), part(hq + hk, hk), slots, n, rng.integers(0, n_pos, T).astype(np.int32), cs


def host(t):
    return t.float().cpu().numpy()


def check_store(hq, hk, d, b, T, dtype, rot, interleaved, norm, seed=0, pad=0, scale=1.0, eps=1e-6):
    rng = np.random.default_rng(seed)
    q, k, v, slots, n, pos, cs = store_case(rng, hq, hk, d, b, T, dtype, rot, pad, scale)
    wq, wk = (dev((1 + 0.2 * rng.standard_normal(d)).astype(np.float32), TYPES[dtype]) for _ in range(2))
    before = K.Cache(n, hk, b, d, rng)
    skip = rng.random(T) < 0.1     # tokens without a slot
    slot = np.where(skip, np.where(rng.random(T) < 0.5, -1, n * b + 3), slots)
    with ctx_of(hq, hk, d, b, n, 4, dtype) as ctx:
        cache = dev(before.bytes)
        out = pkg.kv_store(ctx, q, k, v, dev(pos), dev(slot), cache, dev(cs) if rot else None, rot_dim=rot,
                           interleaved=interleaved, q_weight=wq if norm else None, k_weight=wk if norm else None, eps=eps)
        lk, lv = pkg.kv_load(ctx, cache, dev(slot))
        got = K.Cache(n, hk, b, d)
        got.bytes = cache.cpu().numpy()
    u = UNIT[dtype]
    # queries: 64-bit value, one rounding to 16 bits, and fp32 roundings: the
    # norm's (D/2 + 8 of its sum's terms at most, halved by the root) and two of the rotation's
    want = K.normed_rotated(host(q), host(wq) if norm else None, eps, cs, pos, rot, interleaved)
    size = np.abs(want).max(-1, keepdims=True) * 2 + 1e-30
    tiny = 2.0 ** -25 if dtype == "f16" else 2.0 ** -134
    assert (np.abs(host(out) - want) <= u * np.abs(want) + 16 * 2.0 ** -24 * size + tiny).all()
    # stored: values of the cache
    live = ~skip
    gk, gv = got.get(slot[live])
    code, bits = K.quantised(host(v)[live])
    assert np.array_equal(gv, K.values(code) * (bits.astype(np.uint32) << 16).view(np.float32).astype(np.float64)[..., None])
    want = K.normed_rotated(host(k), host(wk) if norm else None, eps, cs, pos, rot, interleaved)[live]
    s = want.__abs__().max(-1, keepdims=True) / 6
    # the scale is within a bf16 rounding of largest / 6, and no grid value is nearer:
    # half the gap around the value (the top may pass 6 by the scale's rounding)
    a = np.abs(want) / s
    gap = np.where(a < 2, 0.5, np.where(a < 4, 1.0, 2.0))
    assert (np.abs(gk - want) <= (gap / 2 + 6 * 2.0 ** -8 + 1e-5) * s).all()
    _, _, sc = got.parts()
    sk = (sc[slot[live] // b, :, 0, slot[live] % b].astype(np.uint32) << 16).view(np.float32)
    assert (np.abs(sk - s[..., 0]) <= (2.0 ** -8 + 1e-5) * s[..., 0]).all()
    ratio = np.divide(gk, sk[..., None], out=np.zeros_like(gk), where=sk[..., None] != 0)
    near = np.abs(np.abs(want)[..., None] / sk[..., None, None] - np.array([.25, .75, 1.25, 1.75, 2.5, 3.5, 5])).min(-1)
    best = K.values(K.quantised_with(want, sk))
    assert ((ratio == best) | (near < 1e-5)).all()
    # nothing else in the cache changed
    blk, off = slots[live] // b, slots[live] % b
    for x, y, axis in zip(got.parts(), before.parts(), (2, 3, 3)):
        x, y = (np.moveaxis(z, axis, 1).copy() for z in (x, y))
        x[blk, off] = y[blk, off] = 0
        assert np.array_equal(x, y)
    # load gives the same values, rounded; zeros without a slot
    for t, w in ((lk, gk), (lv, gv)):
        t = host(t)
        assert (t[skip] == 0).all()
        assert np.array_equal(t[live], host(torch.from_numpy(w).to(TYPES[dtype])))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("hq,hk,d", [(4, 2, 64), (5, 1, 128), (2, 2, 256)])
def test_store(hq, hk, d, dtype):
    for i, (T, b, rot, inter, norm) in enumerate([(1, 16, d, False, True), (33, 32, d // 2, True, True),
                                                  (70, 64, 16, False, False), (5, 16, 0, False, True),
                                                  (129, 128, d, True, False), (40, 256, d // 4, False, True)]):
        check_store(hq, hk, d, b, T, dtype, rot, inter, norm, seed=i, pad=8 * (i % 3))


@pytest.mark.parametrize("T", [16, 48, 200])
def test_store_runs_of_tokens(T):
    """Prompts: consecutive slots, from an offset inside a block and across blocks."""
    hq, hk, d, b = 4, 2, 128, 32
    rng = np.random.default_rng(T)
    q, k, v, _, n, pos, cs = store_case(rng, hq, hk, d, b, T, "bf16", d)
    for first in (0, 5, 16, 31):
        order = rng.permutation(n + 1)
        slot = np.array([order[(first + i) // b] * b + (first + i) % b for i in range(T)])
        want = K.Cache(n + 1, hk, b, d)
        want.bytes[:] = 170
        cache = dev(want.bytes)
        for t in range(T):
            want.put(slot[t], host(k)[t], host(v)[t])
        with ctx_of(hq, hk, d, b, n + 1, 4) as ctx:
            pkg.kv_store(ctx, q, k, v, dev(pos), dev(slot), cache)
        assert np.array_equal(cache.cpu().numpy(), want.bytes)


def runs_of_slots(rng, T, b, longest):
    """Slots of T tokens: runs of consecutive tokens from anywhere in a block, in blocks of
    any order; a run without slots now and then.  And the number of blocks."""
    slot, used = [], 0
    while len(slot) < T:
        n, first = int(rng.integers(1, longest + 1)), int(rng.integers(0, b))
        n = min(n, T - len(slot))
        if rng.random() < 0.1:
            slot += [-1] * n
        else:
            slot += [used * b + first + i for i in range(n)]
            used += -(-(first + n) // b)
    order = rng.permutation(used)
    slot = np.array(slot)
    return np.where(slot < 0, -1, order[np.maximum(slot, 0) // b] * b + slot % b).astype(np.int64), used


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("hq,hk,d,b,longest", [(12, 4, 64, 16, 300), (14, 1, 128, 32, 40), (9, 3, 256, 64, 700), (16, 2, 128, 16, 3)])
def test_store_many_tokens(hq, hk, d, b, longest, dtype):
    """Large calls: the same bytes and queries, to the last bit, as the tokens a few at a time,
    and values and keys as the oracle's where nothing is normed or rotated."""
    rng = np.random.default_rng(d + b)
    T = 40000 // (hq + 2 * hk) + 13
    q, k, v, _, _, pos, cs = store_case(rng, hq, hk, d, b, T, dtype, d, pad=8)
    slot, n = runs_of_slots(rng, T, b, longest)
    w = dev((1 + 0.2 * rng.standard_normal(d)).astype(np.float32), TYPES[dtype])
    p, sl, c = dev(pos), dev(slot), dev(cs)
    with ctx_of(hq, hk, d, b, n, 4, dtype) as ctx:
        for how in (dict(rot_dim=d, q_weight=w, k_weight=w), dict(rot_dim=d // 2, k_weight=w), dict(rot_dim=d // 4, interleaved=True), dict()):
            table = (c[:, :how["rot_dim"]].contiguous(),) if how.get("rot_dim") else ()
            one, parts = (torch.full((ctx.cache_bytes,), 170, dtype=torch.uint8, device=DEV) for _ in range(2))
            out = pkg.kv_store(ctx, q, k, v, p, sl, one, *table, **how)
            for t in range(0, T, 499):
                e = min(T, t + 499)
                got = pkg.kv_store(ctx, q[t:e], k[t:e], v[t:e], p[t:e].clone(), sl[t:e].clone(), parts, *table, **how)
                assert torch.equal(got, out[t:e]), (how, t)
            assert torch.equal(one, parts), how
    want = K.Cache(n, hk, b, d)
    want.bytes[:] = 170
    hk_, hv_ = host(k), host(v)
    for t in np.nonzero(slot >= 0)[0]:
        want.put(slot[t], hk_[t], hv_[t])
    assert np.array_equal(one.cpu().numpy(), want.bytes.reshape(-1))     # the last: as given
    # read back at once, in any order and from its middle, as a few at a time
    many = np.concatenate([slot, slot[7:], rng.permutation(slot)] * (1 + 65536 // (2 * hk * 3 * T)))
    want_k, want_v = want.get(np.maximum(many, 0))
    with ctx_of(hq, hk, d, b, n, 4, dtype) as ctx:
        for x, y in zip(pkg.kv_load(ctx, one, dev(many)), (want_k, want_v)):
            y[many < 0] = 0
            assert torch.equal(x.cpu(), torch.from_numpy(y).to(TYPES[dtype]))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_store_extremes(dtype):
    """Zeros, one large channel, ties, the type's largest and smallest values,
    infinities and NaN, without norm and rotation: bytes as the oracle's."""
    d, b = 64, 16
    big, small = float(torch.finfo(TYPES[dtype]).max), float(torch.finfo(TYPES[dtype]).smallest_normal)
    x = np.zeros((12, 1, d), np.float32)
    rng = np.random.default_rng(1)
    x[1, 0, 7] = 3
    x[2, 0, :8] = [6, 2.5, 3.5, 5, 0.25, 0.75, -1.75, -1.25]
    x[3] = rng.choice([big, -big, 0, big / 2], (1, d))
    x[4] = rng.choice([small, -small, 0, 2 * small], (1, d))
    x[5] = rng.standard_normal((1, d))
    x[5, 0, 9] = np.inf
    x[6, 0, 0] = -np.inf
    x[7] = rng.standard_normal((1, d))
    x[7, 0, 63] = np.nan
    x[8] = -0.0
    x[9] = rng.standard_normal((1, d)) * 1e-3
    x[10, 0, ::2] = 1
    x[11] = rng.integers(-6, 7, (1, d))
    t = dev(x, TYPES[dtype])
    slot = np.arange(12) + 3
    want = K.Cache(2, 1, b, d)
    with ctx_of(1, 1, d, b, 2, 1, dtype) as ctx:
        cache = dev(want.bytes)
        out = pkg.kv_store(ctx, t, t, t, None, dev(slot), cache)
        k, v = pkg.kv_load(ctx, cache, dev(slot))
    for i in range(12):
        want.put(slot[i], host(t)[i], host(t)[i])
    assert np.array_equal(cache.cpu().numpy(), want.bytes)
    assert np.array_equal(host(out), host(t), equal_nan=True)
    for y in (host(k), host(v)):
        assert np.isnan(y[5:8]).all() and np.isfinite(np.delete(y, [5, 6, 7], 0)).all()


# ---- attention ---------------------------------------------------------------------------------

def attend_case(rng, hq, hk, d, b, rows, dtype, extra=2):
    """rows: (cached, queries, first position or None)."""
    kv = np.array([r[0] for r in rows])
    width = max(1, int((-(-kv // b)).max()))
    n = int((-(-kv // b)).sum()) + extra
    cache = K.Cache(n, hk, b, d)
    cache.bytes[..., :b * d] = rng.integers(0, 256, (n, hk, b * d), dtype=np.uint8)
    s = rng.uniform(0.1, 0.4, (n, hk, 2 * b)).astype(np.float32)
    cache.bytes[..., b * d:] = K.bf16(s)[1].view(np.uint8).reshape(n, hk, 4 * b)
    ids, at = rng.permutation(n).astype(np.int32), 0
    table = np.full((len(rows), width), -1, np.int32)
    q_off, pos = [0], []
    for r, (m, nq, first) in enumerate(rows):
        blocks = -(-m // b)
        table[r, :blocks] = ids[at:at + blocks]
        at += blocks
        q_off.append(q_off[-1] + nq)
        first = m - nq if first is None else first
        pos += list(range(first, first + nq))
    q = rng.standard_normal((q_off[-1], hq, d)).astype(np.float32)
    return (dev(q, TYPES[dtype]), cache, table, kv.astype(np.int32), np.array(q_off, np.int32), np.array(pos, np.int32))


def bound(dtype, want, mag, dots, d, n):
    """|error| of an output: its rounding, the rounding of p * scale (relative u,
    or half the type's smallest step), fp32 products and sums (n terms and the
    exponentials'), and the error of the scores, which multiplies p by at most 1 + 2 delta."""
    u = UNIT[dtype]
    tiny = 6 * n * 2.0 ** -25 if dtype == "f16" else 0.0
    delta = (d + 16) * 2.0 ** -24 * dots[..., None]
    return u * np.abs(want) + (u * 1.01 + 2.2 * delta + (n + 64) * 2.0 ** -23) * mag + tiny + 2.0 ** -25


def check_attend(hq, hk, d, b, rows, dtype="bf16", window=0, seed=0, scale=None, hints=True, pad=0):
    rng = np.random.default_rng(seed)
    q, cache, table, kv, q_off, pos = attend_case(rng, hq, hk, d, b, rows, dtype)
    scale = d ** -0.5 if scale is None else scale
    want, mag, dots = K.attend(host(q), cache, table, kv, q_off, pos, scale, window)
    if pad:   # queries inside a wider buffer
        wide = torch.zeros(len(q), hq * d + pad, dtype=q.dtype, device=DEV)
        wide[:, :hq * d] = q.flatten(1)
        q = wide[:, :hq * d].unflatten(-1, (hq, d))
    nq = max(1, int(np.diff(q_off).max()))
    with ctx_of(hq, hk, d, b, cache.n, table.shape[1], dtype) as ctx:
        args = (ctx, q, dev(cache.bytes), dev(table), dev(kv), dev(q_off), dev(pos))
        every = [(nq, int(kv.max())), (0, 0), (1, 1)] if hints else [(nq, int(kv.max()))]
        for max_q, max_kv in every:
            got = host(pkg.kv_attend(*args, scale=scale, window=window, max_q=max_q, max_kv=max_kv))
            err = np.abs(got - want)
            lim = bound(dtype, want, mag, dots, d, max(1, int(kv.max())))
            assert np.isfinite(got).all()
            assert (err <= lim).all(), (float((err / lim).max()), np.argwhere(err > lim)[:4], max_q, max_kv)
            empty = mag.sum(-1) == 0
            assert (got[empty] == 0).all()


HEADS = [(1, 1, 64), (8, 2, 64), (14, 2, 64), (4, 4, 128), (8, 1, 128), (10, 2, 128), (17, 1, 128), (33, 1, 64), (4, 2, 256)]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("hq,hk,d", HEADS)
def test_attend_single_tokens(hq, hk, d, dtype):
    rows = [(n, 1, None) for n in (1, 2, 15, 16, 17, 63, 64, 65, 130, 257, 0)]
    check_attend(hq, hk, d, 16, rows, dtype, seed=d)


@pytest.mark.parametrize("b", [16, 32, 64, 128, 256])
def test_attend_blocks(b):
    check_attend(8, 2, 128, b, [(n, 1, None) for n in (1, b - 1, b, b + 1, 3 * b + 7, 700)], seed=b)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("hq,hk,d", [(8, 2, 64), (5, 1, 128), (2, 2, 256), (17, 1, 64)])
def test_attend_prompts(hq, hk, d, dtype):
    check_attend(hq, hk, d, 32, [(70, 70, None), (200, 33, None), (1, 1, None), (129, 2, None), (64, 64, None)], dtype, seed=d)


@pytest.mark.parametrize("hq,hk,d,dtype", [(4, 1, 128, "bf16"), (8, 2, 64, "f16"), (6, 3, 256, "bf16"), (7, 1, 64, "bf16")])
def test_attend_long_prompts(hq, hk, d, dtype):
    """Several tiles of columns a row and many steps of tokens, with and without a window."""
    rows = [(700, 700, None), (390, 130, None), (64, 64, None), (0, 5, 0), (1000, 90, None)]
    check_attend(hq, hk, d, 32, rows, dtype, seed=d + hq)
    check_attend(hq, hk, d, 16, rows, dtype, seed=d + hq, window=150, hints=False)


@pytest.mark.parametrize("window", [1, 2, 16, 63, 64, 100, 5000])
def test_attend_window(window):
    check_attend(8, 2, 64, 16, [(300, 1, None), (150, 90, None), (40, 40, None), (1, 1, None)], window=window, seed=window)


def test_attend_empty_rows():
    """Rows without cached tokens (refused), positions before the first token and
    past the last, rows without queries."""
    check_attend(8, 2, 128, 16, [(0, 3, 0), (5, 9, -4), (50, 0, None), (20, 4, 18), (0, 0, 0), (33, 5, 60), (7, 1, -1)],
                 window=0, seed=1)
    check_attend(8, 2, 128, 16, [(20, 6, 18), (33, 5, 60), (40, 3, -1)], window=4, seed=2)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_attend_longer(dtype):
    check_attend(8, 2, 128, 64, [(5000, 1, None), (1100, 1, None), (3, 1, None)], dtype, seed=7)
    check_attend(4, 1, 64, 16, [(2100, 17, None), (900, 1, None)], dtype, seed=8)


def test_attend_large_scores():
    # one token takes nearly all the weight; negative and zero scales
    for scale in (4.0, -1.0, 0.0):
        check_attend(8, 2, 64, 16, [(500, 1, None), (60, 20, None)], scale=scale, seed=3)


def test_attend_strided_queries():
    check_attend(8, 2, 64, 16, [(90, 1, None), (60, 5, None)], pad=24, seed=4, hints=False)


def test_attend_many_rows():
    rng = np.random.default_rng(9)
    check_attend(4, 2, 64, 16, [(int(n), 1, None) for n in rng.integers(0, 90, 300)], seed=9)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_attend_masked_garbage_does_not_leak(dtype):
    """NaN and infinite scales past a row's end, before its window, and in blocks of
    no row; ids of unused table entries out of range."""
    hq, hk, d, b, window = 8, 2, 64, 16, 50
    rng = np.random.default_rng(11)
    rows = [(37, 1, None), (100, 1, None), (90, 13, None), (0, 1, 0)]
    q, cache, table, kv, q_off, pos = attend_case(rng, hq, hk, d, b, rows, dtype)
    want, mag, dots = K.attend(host(q), cache, table, kv, q_off, pos, d ** -0.5, window)
    raw = cache.bytes[..., b * d:].copy().view(np.uint16).reshape(cache.n, hk, 2, b)
    seen = np.zeros((cache.n, b), bool)
    for r, (n, nq, _) in enumerate(rows):
        for j in range(max(0, n - nq - window + 1), n):
            seen[table[r, j // b], j % b] = True
    bad = rng.choice(np.array([0x7fc0, 0x7f80, 0xff80, 0x7f7f], np.uint16), raw.shape)
    raw = np.where(seen[:, None, None, :], raw, bad)
    cache.bytes[..., b * d:] = np.ascontiguousarray(raw).view(np.uint8).reshape(cache.n, hk, 4 * b)
    table = np.where(table < 0, rng.choice(np.array([-1, 2 ** 31 - 1, -2 ** 31, cache.n], np.int32), table.shape), table).astype(np.int32)
    with ctx_of(hq, hk, d, b, cache.n, table.shape[1], dtype) as ctx:
        got = host(pkg.kv_attend(ctx, q, dev(cache.bytes), dev(table), dev(kv), dev(q_off), dev(pos), scale=d ** -0.5, window=window))
    assert (np.abs(got - want) <= bound(dtype, want, mag, dots, d, 100)).all()


def test_attend_nan_in_sight_shows():
    """A stored NaN reaches the queries that see it, and no others."""
    hq, hk, d, b = 4, 2, 64, 16
    rng = np.random.default_rng(12)
    q, cache, table, kv, q_off, pos = attend_case(rng, hq, hk, d, b, [(40, 40, None)], "bf16")
    cell = cache.bytes[table[0, 1], 1]                 # token 20 of kv head 1: its key
    cell[b * d:].view(np.uint16)[4] = 0x7fc0
    with ctx_of(hq, hk, d, b, cache.n, table.shape[1]) as ctx:
        got = host(pkg.kv_attend(ctx, q, dev(cache.bytes), dev(table), dev(kv), dev(q_off), dev(pos), scale=0.125))
    assert np.isnan(got[20:, 2:]).all()
    assert np.isfinite(got[:20]).all() and np.isfinite(got[:, :2]).all()


def skewed_case(rng, hq, hk, d, b, n, nq, dtype, far, size=1.0):
    """nq queries of one row over n tokens; the tokens in `far` have large keys along the queries'
    common direction, all others small ones; value scales `size` times the usual."""
    q, cache, table, kv, q_off, pos = attend_case(rng, hq, hk, d, b, [(n, nq, None)], dtype)
    x = 0.1 * rng.standard_normal((n, hk, d)).astype(np.float32)
    line = rng.standard_normal(d).astype(np.float32)
    for j, f in far.items():
        x[j] = f * line
    q = dev((line + 0.1 * rng.standard_normal((nq, hq, d))).astype(np.float32), TYPES[dtype])
    v = (size * rng.standard_normal((n, hk, d))).astype(np.float32)
    for j in range(n):
        cache.put(int(table[0, j // b]) * b + j % b, x[j], v[j])
    return q, cache, table, kv, q_off, pos


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("hq,hk,d", [(8, 1, 64), (4, 1, 128), (6, 1, 256)])
def test_attend_prompts_of_uneven_scores(hq, hk, d, dtype):
    """Many columns whose largest score is far above or below those of the last and the first
    tokens: at one early token, in the middle, at the end only; large and small values."""
    b, n, nq = 16, 450, 60
    for i, (far, size) in enumerate([({3: 8.0}, 1.0), ({200: 20.0}, 1.0), ({449: 30.0}, 1.0), ({0: -20.0, 447: -20.0}, 1.0),
                                     ({5: 3.0, 300: 3.0}, 400.0), ({100: 12.0}, 3000.0), ({}, 0.01)]):
        rng = np.random.default_rng(100 * i + d)
        q, cache, table, kv, q_off, pos = skewed_case(rng, hq, hk, d, b, n, nq, dtype, far, size)
        want, mag, dots = K.attend(host(q), cache, table, kv, q_off, pos, d ** -0.5, 0)
        with ctx_of(hq, hk, d, b, cache.n, table.shape[1], dtype) as ctx:
            both = [host(pkg.kv_attend(ctx, q, dev(cache.bytes), dev(table), dev(kv), dev(q_off), dev(pos), scale=d ** -0.5,
                                       **hints)) for hints in (dict(max_q=nq, max_kv=n), dict())]
        # as bound(); for f16, a probability times its value scale is rounded to a step of 2^-25 of a
        # total that may be as small as 2^-8 (the reference is within 8 powers of two of the largest score)
        lim = bound(dtype, want, mag, dots, d, n) + (6 * n * 2.0 ** -17 if dtype == "f16" else 0.0)
        for got in both:
            assert np.isfinite(got).all(), i
            assert (np.abs(got - want) <= lim).all(), (i, float((np.abs(got - want) / lim).max()))


def test_floats_are_not_taken_for_integers():
    with ctx_of(4, 2, 64, 16, 8, 4) as ctx:
        x = lambda *s, dt=torch.bfloat16: torch.zeros(*s, dtype=dt, device=DEV)
        cache, q, k, slot = x(ctx.cache_bytes, dt=torch.uint8), x(3, 4, 64), x(3, 2, 64), x(3, dt=torch.int64)
        for bad in (dict(pos=x(3, dt=torch.float32)), dict(slot=slot.double()), dict(cos_sin=x(4, 64, dt=torch.int32), rot_dim=64)):
            with pytest.raises(TypeError):
                how = {**dict(pos=x(3, dt=torch.int32), slot=slot, cos_sin=x(4, 64, dt=torch.float32), rot_dim=64), **bad}
                pkg.kv_store(ctx, q, k, k, how["pos"], how["slot"], cache, how["cos_sin"], rot_dim=64)


@pytest.mark.parametrize("hq,hk,rows", [(128, 128, 40000), (8, 2, 65536)])
def test_attend_more_rows_than_one_grid(hq, hk, rows):
    """Batches whose workgroups do not fit one grid: each row has its own token's value."""
    d, b = 64, 16
    rng = np.random.default_rng(rows)
    x = torch.from_numpy(rng.integers(-6, 7, (32, hk, d)).astype(np.float32)).to(DEV).bfloat16()
    x[..., 0] = 6                                          # scale 1: integers up to 6 less the ones off the grid
    slots = torch.arange(32, device=DEV) * b               # 32 blocks of one token
    with ctx_of(hq, hk, d, b, 32, 1) as ctx:
        cache = torch.zeros(ctx.cache_bytes, dtype=torch.uint8, device=DEV)
        pkg.kv_store(ctx, x[:, :1].expand(32, hq, d).contiguous(), x, x, None, slots, cache)
        _, v = pkg.kv_load(ctx, cache, slots)
        at = torch.arange(rows, device=DEV) % 32
        ones = torch.ones(rows, dtype=torch.int32, device=DEV)
        q = torch.ones(1, hq, d, dtype=torch.bfloat16, device=DEV).expand(rows, hq, d).contiguous()
        for hint in (1, 0):                                # 0: as many columns a row as there are tokens
            out = pkg.kv_attend(ctx, q, cache, at.int()[:, None].contiguous(), ones, torch.arange(rows + 1, device=DEV).int(), ones - 1,
                                scale=1.0, max_q=hint, max_kv=1)
            assert torch.equal(out.view(rows, hk, hq // hk, d), v[at][:, :, None].expand(-1, -1, hq // hk, -1))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("hq,hk,d,b", [(8, 2, 64, 16), (4, 1, 128, 64), (4, 2, 256, 32)])
def test_attend_prompts_beside_garbage(hq, hk, d, b, dtype):
    """Many columns: NaN and infinite scales past a row's end, before its window, in other blocks."""
    rng = np.random.default_rng(d)
    window, rows = 90, [(333, 80, None), (70, 70, None), (0, 40, 0), (200, 45, None)]
    q, cache, table, kv, q_off, pos = attend_case(rng, hq, hk, d, b, rows, dtype)
    want, mag, dots = K.attend(host(q), cache, table, kv, q_off, pos, d ** -0.5, window)
    raw = cache.bytes[..., b * d:].copy().view(np.uint16).reshape(cache.n, hk, 2, b)
    seen = np.zeros((cache.n, b), bool)
    for r, (n, nq, _) in enumerate(rows):
        for j in range(max(0, n - nq - window + 1), n):
            seen[table[r, j // b], j % b] = True
    raw = np.where(seen[:, None, None, :], raw, rng.choice(np.array([0x7fc0, 0x7f80, 0xff80, 0x7f7f], np.uint16), raw.shape))
    cache.bytes[..., b * d:] = np.ascontiguousarray(raw).view(np.uint8).reshape(cache.n, hk, 4 * b)
    with ctx_of(hq, hk, d, b, cache.n, table.shape[1], dtype) as ctx:
        for hints in (dict(max_q=80, max_kv=333), dict()):
            got = host(pkg.kv_attend(ctx, q, dev(cache.bytes), dev(table), dev(kv), dev(q_off), dev(pos), scale=d ** -0.5,
                                     window=window, **hints))
            assert (np.abs(got - want) <= bound(dtype, want, mag, dots, d, window)).all()


@pytest.mark.parametrize("hq,hk,d,nq", [(8, 1, 64, 3), (8, 1, 128, 16), (16, 1, 128, 20), (4, 1, 256, 90)])
def test_attend_few_queries_over_many_tokens(hq, hk, d, nq):
    """One row in many shares, joined by the last workgroup or by a launch of its own."""
    check_attend(hq, hk, d, 64, [(9000, nq, None)], seed=nq)
    check_attend(hq, hk, d, 64, [(2500, nq, None), (700, 1, None)], "f16", seed=nq)
    check_attend(hq, hk, d, 64, [(600, nq, None), (400, nq, None), (1300, 3, None)], "f16", seed=nq, window=450)


def test_attend_cache_past_32_bits():
    """Blocks whose bytes lie past 2^32: the first and the last block of a 5 GiB cache."""
    hq, hk, d, b = 8, 8, 128, 64
    n = (5 << 30) // (hk * b * (d + 4)) + 1
    rng = np.random.default_rng(13)
    q, small, table, kv, q_off, pos = attend_case(rng, hq, hk, d, b, [(100, 1, None)], "bf16", extra=0)
    want, mag, dots = K.attend(host(q), small, table, kv, q_off, pos, d ** -0.5, 0)
    with ctx_of(hq, hk, d, b, n, 2) as ctx:
        cache = torch.zeros(ctx.cache_bytes, dtype=torch.uint8, device=DEV).view(n, hk, -1)
        cache[n - 1], cache[0] = dev(small.bytes[table[0, 0]]), dev(small.bytes[table[0, 1]])
        far = dev(np.array([[n - 1, 0]], np.int32))
        got = host(pkg.kv_attend(ctx, q, cache, far, dev(kv), dev(q_off), dev(pos), scale=d ** -0.5))
        assert (np.abs(got - want) <= bound("bf16", want, mag, dots, d, 100)).all()
        # stored and read back there
        x = dev(rng.standard_normal((2, hk, d)).astype(np.float32), torch.bfloat16)
        slot = dev(np.array([n * b - 1, (n - 1) * b + 3]))
        pkg.kv_store(ctx, x, x, x, None, slot, cache)
        k, v = pkg.kv_load(ctx, cache, slot)
        for t in (k, v):
            code, bits = K.quantised(host(x))
            w = K.values(code) * (bits.astype(np.uint32) << 16).view(np.float32)[..., None]
            assert np.array_equal(host(t), host(torch.from_numpy(w).to(torch.bfloat16)))


# ---- calls -------------------------------------------------------------------------------------

def test_streams_and_replays():
    """On a stream of its own and replayed from a graph: the eager results."""
    rng = np.random.default_rng(21)
    hq, hk, d, b = 8, 2, 128, 16
    q, cache, table, kv, q_off, pos = attend_case(rng, hq, hk, d, b, [(900, 1, None), (70, 1, None), (333, 5, None)], "bf16")
    with ctx_of(hq, hk, d, b, cache.n, table.shape[1]) as ctx:
        c, tb, ln, qo, ps = dev(cache.bytes), dev(table), dev(kv), dev(q_off), dev(pos)
        run = lambda x, **kw: pkg.kv_attend(ctx, x, c, tb, ln, qo, ps, scale=d ** -0.5, max_q=5, max_kv=900, **kw)
        q2 = torch.roll(q, 1, 0)
        eager = [run(x).clone() for x in (q, q2)]
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            side = run(q)
        side2 = run(q, stream=s)
        torch.cuda.synchronize()
        assert torch.equal(side, eager[0]) and torch.equal(side2, eager[0])
        x, out = q.clone(), torch.empty_like(q)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            ctx.wf_kv_attend(x, len(x), c, tb, ln, qo, ps, 3, d ** -0.5, out, max_q=5, max_kv=900)
        for k in range(6):
            x.copy_((q, q2)[k % 2])
            run(q2 if k % 2 == 0 else q)              # eager work of the same context between
            out.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, eager[k % 2]), k


@pytest.mark.parametrize("prompt", [1, 90])
def test_a_whole_step_replays(prompt):
    """Step, store, attention and load in one graph, replayed with other keys, values and queries: what
    the same calls give one after the other."""
    rng = np.random.default_rng(41)
    hq, hk, d, b, rows, width = 8, 2, 64, 16, 12, 40
    lens = rng.integers(0, 400, rows).astype(np.int32)
    new = np.where(rng.random(rows) < 0.3, prompt, 1).astype(np.int32)
    new[3] = -1
    have = -(-lens // b)
    n = int(have.sum()) + rows * (1 + prompt // b)
    ids, at, table = rng.permutation(n).astype(np.int32), 0, np.full((rows, width), -1, np.int32)
    for r in range(rows):
        table[r, :have[r]] = ids[at:at + have[r]]
        at += have[r]
    ring = np.roll(np.concatenate([ids[at:], np.full(at, -1, np.int32)]), 7)
    T = int(np.maximum(new, 0).sum())
    raw = K.Cache(n, hk, b, d, rng).bytes
    raw[..., b * d:] = K.bf16(rng.uniform(0.1, 0.4, (n, hk, 2 * b)).astype(np.float32))[1].view(np.uint8).reshape(n, hk, 4 * b)
    inputs = [[dev(rng.standard_normal((T, h, d)).astype(np.float32), torch.bfloat16) for h in (hq, hk, hk)] for _ in range(2)]
    cs = torch.rand(width * b, d, device=DEV)
    with ctx_of(hq, hk, d, b, n, width) as ctx:
        fresh, ln, pool = dev(new), dev(lens), dev(np.array([7, n - at], np.int32))

        def step(qkv, cache, rg, tb):
            out_lens, out_pool, q_off, slot, pos, granted = pkg.kv_step(ctx, fresh, T, ln, pool, rg, tb)
            q = pkg.kv_store(ctx, *qkv, pos, slot, cache, cs, rot_dim=d)
            o = pkg.kv_attend(ctx, q, cache, tb, out_lens, q_off, pos, scale=0.125, max_q=prompt, max_kv=500)
            return [out_lens, out_pool, q_off, slot, pos, granted, q, o, *pkg.kv_load(ctx, cache, slot), cache, rg, tb]
        eager = [[x.clone() for x in step(qkv, dev(raw), dev(ring), dev(table))] for qkv in inputs]
        held, cache, rg, tb = [x.clone() for x in inputs[0]], dev(raw), dev(ring), dev(table)
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph):
            out = step(held, cache, rg, tb)
        for k in range(6):
            for x, y in zip((*held, cache, rg, tb), (*inputs[k % 2], dev(raw), dev(ring), dev(table))):
                x.copy_(y)
            step(inputs[1 - k % 2], dev(raw), dev(ring), dev(table))     # eager work of the same context between
            graph.replay()
            torch.cuda.synchronize()
            for i, (x, y) in enumerate(zip(out, eager[k % 2])):
                assert torch.equal(x, y), (k, i)


@pytest.mark.parametrize("handle", [False, True])
def test_outputs_belong_to_the_stream(handle):
    """Outputs of a call on a given stream are that stream's memory: once dropped, the current
    stream does not get it while the other may still write it."""
    with ctx_of(4, 2, 64, 16, 8, 4) as ctx:
        slot = torch.arange(64, device=DEV)
        cache = torch.zeros(ctx.cache_bytes, dtype=torch.uint8, device=DEV)
        off, lens = torch.tensor([0, 64], dtype=torch.int32, device=DEV), torch.tensor([64], dtype=torch.int32, device=DEV)
        table, q = torch.arange(4, dtype=torch.int32, device=DEV)[None], torch.ones(64, 4, 64, dtype=torch.bfloat16, device=DEV)
        kv = q[:, :2].contiguous()
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        on = dict(stream=s.cuda_stream if handle else s)
        for call in (lambda: pkg.kv_load(ctx, cache, slot, **on)[0], lambda: pkg.kv_store(ctx, q, kv, kv, None, slot, cache, **on),
                     lambda: pkg.kv_attend(ctx, q, cache, table, lens, off, slot.int(), scale=0.125, **on),
                     lambda: pkg.kv_step(ctx, lens, 64, lens, off[:2].clone(), torch.arange(8, dtype=torch.int32, device=DEV),
                                         table.clone(), **on)[3]):
            out = call()
            shape, kind, at = out.shape, out.dtype, out.data_ptr()
            del out
            assert torch.empty(shape, dtype=kind, device=DEV).data_ptr() != at
            with torch.cuda.stream(s):
                assert abs(torch.empty(shape, dtype=kind, device=DEV).data_ptr() - at) < 2 << 20    # its segment
        torch.cuda.synchronize()


def test_both_ways_of_a_call_agree(monkeypatch):
    """The helpers through _kvbind and through ctypes: the same outputs, the same refusals."""
    rng = np.random.default_rng(31)
    hq, hk, d, b = 8, 2, 64, 16
    q, cache, table, kv, q_off, pos = attend_case(rng, hq, hk, d, b, [(90, 3, None), (40, 1, None), (17, 17, None)], "bf16")
    lens, new, tb, ring, pool = random_step(rng, 70, b, table.shape[1], 0.7)
    with ctx_of(hq, hk, d, b, cache.n, table.shape[1]) as ctx, ctx_of(hq, hk, d, b, len(ring), table.shape[1]) as sctx:
        assert ctx._bind is not None, "_kvbind is not built"
        c, x = dev(cache.bytes), dev(rng.standard_normal((21, hk, d)).astype(np.float32), torch.bfloat16)
        w, cs = torch.ones(d, dtype=torch.bfloat16, device=DEV), torch.rand(99, d, device=DEV)
        slot, p = dev(rng.permutation(cache.n * b)[:21]), dev(pos)
        tokens = int(np.maximum(new, 0).sum())

        def calls():
            mine, r, t = c.clone(), dev(ring), dev(tb)
            return [pkg.kv_attend(ctx, q, c, dev(table), dev(kv), dev(q_off), p, scale=0.125, window=20, max_q=17, max_kv=90),
                    pkg.kv_store(ctx, q, x, x, p, slot, mine, cs, rot_dim=d, q_weight=w), mine, *pkg.kv_load(ctx, c, slot),
                    *pkg.kv_step(sctx, dev(new), tokens, dev(lens), dev(pool), r, t), r, t]
        bad = [(lambda: pkg.kv_load(ctx, c, slot.int()), TypeError), (lambda: pkg.kv_load(ctx, c.cpu(), slot), ValueError),
               (lambda: pkg.kv_load(ctx, c.flatten()[:-1], slot), ValueError),
               (lambda: pkg.kv_store(ctx, q, x[:-1], x, p, slot, c), ValueError),
               (lambda: pkg.kv_store(ctx, q.half(), x, x, p, slot, c), TypeError),
               (lambda: pkg.kv_store(ctx, q, x, x, p, slot, c, eps=-1.0), pkg.WFError),
               (lambda: pkg.kv_attend(ctx, q, c, dev(table), dev(kv), dev(q_off), p, scale=float("nan")), pkg.WFError),
               (lambda: pkg.kv_attend(ctx, q, c, dev(table), dev(kv), dev(q_off), p, scale=0.1, window=-1), pkg.WFError),
               (lambda: pkg.kv_step(sctx, dev(new), -1, dev(lens), dev(pool), dev(ring), dev(tb)), (pkg.WFError, RuntimeError)),
               (lambda: pkg.kv_step(sctx, dev(new), tokens, dev(lens)[:-1], dev(pool), dev(ring), dev(tb)), ValueError)]
        results = []
        for way in (ctx._bind, None):
            monkeypatch.setattr(ctx, "_bind", way)
            monkeypatch.setattr(sctx, "_bind", way)
            results.append(calls())
            for call, error in bad:
                with pytest.raises(error):
                    call()
        assert len(results[0]) == len(results[1]) == 13
        for one, two in zip(*results):
            assert one.shape == two.shape and one.dtype == two.dtype and torch.equal(one, two)
        # addresses, an integer scale and a 2-D view go the longer way
        monkeypatch.undo()
        assert torch.equal(pkg.kv_attend(ctx, q.flatten(1), c, dev(table), dev(kv), dev(q_off), p, scale=1),
                           pkg.kv_attend(ctx, q, c, dev(table), dev(kv), dev(q_off), p, scale=1.0))
    with pytest.raises(pkg.WFError):
        pkg.kv_load(ctx, c, slot)                          # closed


def test_refusals():
    hq, hk, d, b = 4, 2, 64, 16
    with ctx_of(hq, hk, d, b, 8, 4) as ctx:
        x = lambda *s, dt=torch.bfloat16: torch.zeros(*s, dtype=dt, device=DEV)
        i32, i64 = torch.int32, torch.int64
        cache, q, k, slot, pos = x(ctx.cache_bytes, dt=torch.uint8), x(3, hq, d), x(3, hk, d), x(3, dt=i64), x(3, dt=i32)
        store = lambda **kw: ctx.wf_kv_store(**{**dict(q=q, k=k, v=k, n_tokens=3, pos=pos, slot=slot, q_out=x(3, hq, d), cache=cache), **kw})
        store()
        for bad in (dict(q=q.cpu()), dict(q=x(2, hq, d)), dict(q=x(3, hq, d, dt=torch.float16)), dict(q=x(3, hk, d)),
                    dict(k=x(3, hk, 2 * d)[..., ::2]), dict(v=k.transpose(1, 2)), dict(slot=x(2, dt=i64)),
                    dict(slot=x(3, dt=i32)), dict(cache=cache[:-1]), dict(q_out=x(2, hq, d)), dict(pos=x(3, dt=i64)),
                    dict(q_weight=x(d - 1)), dict(cos_sin=x(4, 16, dt=torch.float32), n_pos=5, rot_dim=16)):
            with pytest.raises((ValueError, TypeError)):
                store(**bad)
        cs = x(4, 64, dt=torch.float32)
        for bad in (dict(n_tokens=-1), dict(rot_dim=8, cos_sin=cs, n_pos=4), dict(rot_dim=80, cos_sin=cs, n_pos=1),
                    dict(rot_dim=16), dict(rot_dim=16, cos_sin=cs, n_pos=0), dict(rot_dim=16, cos_sin=cs, n_pos=4, pos=None),
                    dict(eps=-1.0), dict(eps=float("nan")), dict(slot=None), dict(q=None), dict(cache=None),
                    dict(q=x(4 * 3 * hq * d)[4:][:3 * hq * d].view(3, hq, d)),           # 8 bytes off
                    dict(k=x(3, hk * d + 4)[:, :hk * d].unflatten(-1, (hk, d)))):         # stride not a multiple of 8
            with pytest.raises(pkg.WFError) as e:
                store(**bad)
            assert e.value.status == pkg.WF_EINVAL and e.value.message
        table, lens, off = x(2, 4, dt=i32), x(2, dt=i32), x(3, dt=i32)
        att = lambda **kw: ctx.wf_kv_attend(**{**dict(q=q, n_tokens=3, cache=cache, table=table, kv_len=lens, q_off=off, pos=pos,
                                                      n_rows=2, scale=1.0, out=x(3, hq, d)), **kw})
        att()
        for bad in (dict(table=x(2, 3, dt=i32)), dict(kv_len=x(1, dt=i32)), dict(q_off=x(2, dt=i32)), dict(out=x(3, hk, d)),
                    dict(q=q.float()), dict(pos=pos.long()), dict(table=table.cpu())):
            with pytest.raises((ValueError, TypeError)):
                att(**bad)
        for bad in (dict(n_rows=-1), dict(n_tokens=-2), dict(window=-1), dict(max_q=-1), dict(max_kv=-1), dict(table=None),
                    dict(scale=float("inf")), dict(scale=float("nan")), dict(out=None)):
            with pytest.raises(pkg.WFError) as e:
                att(**bad)
            assert e.value.status == pkg.WF_EINVAL
        att(n_tokens=0)
        att(n_rows=0)
        new, pool, pool2, ring = x(2, dt=i32), x(2, dt=i32), x(2, dt=i32), x(8, dt=i32)
        stp = lambda **kw: ctx.wf_kv_step(**{**dict(new_tokens=new, n_rows=2, n_tokens=3, len_in=lens, len_out=x(2, dt=i32), pool_in=pool,
                                                    pool_out=pool2, ring=ring, table=table, q_off=off, slot=slot, pos=pos,
                                                    granted=x(2, dt=torch.uint8)), **kw})
        stp()
        for bad in (dict(ring=x(7, dt=i32)), dict(q_off=x(2, dt=i32)), dict(slot=x(2, dt=i64)), dict(new_tokens=new.long())):
            with pytest.raises((ValueError, TypeError)):
                stp(**bad)
        for bad in (dict(n_rows=-1), dict(n_tokens=-1), dict(n_rows=1 << 17, new_tokens=0, len_in=0, len_out=0, table=0, granted=0, q_off=0),
                    dict(len_out=lens), dict(pool_out=pool), dict(new_tokens=None), dict(slot=None)):
            with pytest.raises(pkg.WFError) as e:
                stp(**bad)
            assert e.value.status == pkg.WF_EINVAL
        with pytest.raises(pkg.WFError):
            ctx.wf_kv_load(cache, slot, -1, k, k)
        with pytest.raises(pkg.WFError):
            ctx.wf_kv_load(cache, None, 3, k, k)
        torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("hq,hk,d", [(8, 2, 64), (4, 2, 128), (4, 2, 256)])
def test_attend_positions_past_every_window(hq, hk, d, dtype):
    """Positions as far as the largest integer, for rows of any length: nothing is seen through a window, the whole
    row without one; by the kernel of few columns and by that of many, among sound queries of the same call."""
    rng = np.random.default_rng(d)
    top = 2 ** 31 - 1
    for queries in (1, 70):
        rows = [(90, queries, None), (300, queries, None), (0, queries, 0), (40, queries, -queries)]
        q, cache, table, kv, q_off, pos = attend_case(rng, hq, hk, d, 16, rows, dtype)
        far = pos.copy()
        far[:q_off[2]] = top - np.arange(q_off[2]) % 3 * 300
        mixed = np.where(np.arange(len(pos)) % 2 == 0, far, pos)
        with ctx_of(hq, hk, d, 16, cache.n, table.shape[1], dtype) as ctx:
            for p in (far, mixed):
                for window in (0, 1, 64, top):
                    want, mag, dots = K.attend(host(q), cache, table, kv, q_off, p.astype(np.int64), d ** -0.5, window)
                    for hints in (dict(max_q=queries, max_kv=300), dict()):
                        got = host(pkg.kv_attend(ctx, q, dev(cache.bytes), dev(table), dev(kv), dev(q_off), dev(p.astype(np.int32)),
                                                 scale=d ** -0.5, window=window, **hints))
                        assert (np.abs(got - want) <= bound(dtype, want, mag, dots, d, 300)).all(), (queries, window)
                        assert (got[mag.sum(-1) == 0] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("hq,hk,d", [(8, 1, 64), (4, 1, 128), (4, 1, 256)])
def test_attend_is_as_accurate_for_small_and_large_values(hq, hk, d, dtype):
    """Values of sizes 2^-13 to 2^11, one score 10 powers of two above a long tail of others or none, by the kernels
    of 16, of 32 and of many columns: the error is bounded relative to the values."""
    b, n, most = 16, 1500, 70
    u = UNIT[dtype]
    for i, at in enumerate((None, 7, n - 1)):
        far = {} if at is None else {at: 10 / (1.4427 * d ** 0.5)}
        q, cache, table, kv, q_off, pos = skewed_case(np.random.default_rng(10 * d + i), hq, hk, d, b, n, most, dtype, far)
        want, mag, dots = K.attend(host(q), cache, table, kv, q_off, pos, d ** -0.5, 0)
        with ctx_of(hq, hk, d, b, cache.n, table.shape[1], dtype) as ctx:
            for power in (0, -7, -10, -13, 11):
                raw, size = cache.bytes.copy(), 2.0 ** power
                raw[..., b * d:].view(np.uint16)[..., b:] += np.uint16((power << 7) & 0xffff)      # scales of the values
                for nq in (1, 5, most):
                    got = host(pkg.kv_attend(ctx, q[-nq:], dev(raw), dev(table), dev(kv), dev(np.array([0, nq], np.int32)),
                                             dev(pos[-nq:].copy()), scale=d ** -0.5, max_q=nq, max_kv=n))
                    w, m = want[-nq:] * size, mag[-nq:] * size
                    # as in bound(), but for f16's small steps: a probability times a value scale is rounded to half a step,
                    # 2^-25, of a number whose largest is at least 2^-2; a scale is a sixth of some channel
                    delta = (d + 16) * 2.0 ** -24 * dots[-nq:][..., None]
                    lim = u * np.abs(w) + (1.01 * u + 2.2 * delta + (n + 64) * 2.0 ** -23) * m + 2.0 ** -25
                    if dtype == "f16":
                        lim += n * 2.0 ** -23 * m.max(-1, keepdims=True)
                    assert (np.abs(w) > lim).any(-1).all()        # zeros would not pass
                    assert (np.abs(got - w) <= lim).all(), (at, power, nq, float((np.abs(got - w) / lim).max()))


@pytest.mark.parametrize("hq,hk,d", [(8, 1, 64), (4, 1, 128), (4, 1, 256)])
def test_attend_uneven_values(hq, hk, d):
    """f16: the token that has most of the weight with a value of zeros, and one of next to no weight with a value a
    thousand times the others', by the kernels of 16, of 32 and of many columns."""
    b, n, most = 16, 700, 70
    one = 1 / (1.4427 * d ** 0.5)                                # a power of two in the score
    for i, (sink, loud) in enumerate(((None, 400), (7, None), (690, 3), (3, 690))):
        far = {**({} if sink is None else {sink: 20 * one}), **({} if loud is None else {loud: -12 * one})}
        q, cache, table, kv, q_off, pos = skewed_case(np.random.default_rng(5 * d + i), hq, hk, d, b, n, most, "f16", far, 8.0)
        for j, size in ((sink, 0.0), (loud, 8000.0)):
            if j is not None:
                keys, _ = cache.get([int(table[0, j // b]) * b + j % b])
                cache.put(int(table[0, j // b]) * b + j % b, keys[0].astype(np.float32),
                          (size * np.random.default_rng(j).uniform(0.5, 1, (hk, d))).astype(np.float32))
        want, mag, dots = K.attend(host(q), cache, table, kv, q_off, pos, d ** -0.5, 0)
        with ctx_of(hq, hk, d, b, cache.n, table.shape[1], "f16") as ctx:
            for nq in (1, 5, most):
                got = host(pkg.kv_attend(ctx, q[-nq:], dev(cache.bytes), dev(table), dev(kv), dev(np.array([0, nq], np.int32)),
                                         dev(pos[-nq:].copy()), scale=d ** -0.5, max_q=nq, max_kv=n))
                w, m, u = want[-nq:], mag[-nq:], UNIT["f16"]
                # as in the test before
                lim = u * np.abs(w) + (1.01 * u + 2.2 * (d + 16) * 2.0 ** -24 * dots[-nq:][..., None] + (n + 64) * 2.0 ** -23) * m
                lim += 2.0 ** -25 + n * 2.0 ** -23 * m.max(-1, keepdims=True)
                assert (np.abs(w) > lim).any(-1).all()
                assert (np.abs(got - w) <= lim).all(), (sink, loud, nq, float((np.abs(got - w) / lim).max()))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("window", [1, 2, 16, 63, 100])
def test_attend_prompts_through_small_windows(window, dtype):
    """Many columns whose windows share no tokens, some or all."""
    check_attend(8, 2, 64, 16, [(300, 200, None), (150, 90, None), (40, 40, None)], dtype, window=window, seed=window)
    check_attend(3, 3, 128, 32, [(400, 300, None)], dtype, window=window, seed=window)


def test_attend_over_zeros():
    """A cache of zeros, as it may be before its first use."""
    for hq, hk, d in ((8, 1, 64), (4, 1, 128), (4, 1, 256)):
        for dtype in ("bf16", "f16"):
            with ctx_of(hq, hk, d, 16, 32, 32, dtype) as ctx:
                q = torch.randn(60, hq, d, device=DEV).to(TYPES[dtype])
                table, pos = torch.arange(32, dtype=torch.int32, device=DEV)[None], torch.arange(440, 500, dtype=torch.int32, device=DEV)
                cache = torch.zeros(ctx.cache_bytes, dtype=torch.uint8, device=DEV)
                for nq in (1, 5, 60):
                    off, kv = dev(np.array([0, nq], np.int32)), dev(np.array([500], np.int32))
                    out = pkg.kv_attend(ctx, q[:nq], cache, table, kv, off, pos[:nq].clone(), scale=0.1, max_q=nq, max_kv=500)
                    assert (out == 0).all()


def test_rows_of_another_length_are_refused(monkeypatch):
    """Block tables wider or narrower than the context's and rotations of other channels, with as many elements
    as are needed or more: refused by both ways of a call, before anything is written."""
    hq, hk, d, b, width, rows = 4, 2, 64, 16, 4, 3
    i32 = torch.int32
    with ctx_of(hq, hk, d, b, 32, width) as ctx:
        cache = torch.zeros(ctx.cache_bytes, dtype=torch.uint8, device=DEV)
        q, k = torch.ones(rows, hq, d, dtype=torch.bfloat16, device=DEV), torch.ones(rows, hk, d, dtype=torch.bfloat16, device=DEV)
        ones, off, pos = torch.ones(rows, dtype=i32, device=DEV), torch.arange(rows + 1, dtype=i32, device=DEV), torch.zeros(rows, dtype=i32, device=DEV)
        ring, pool, slot = torch.arange(32, dtype=i32, device=DEV), torch.tensor([0, 32], dtype=i32, device=DEV), torch.arange(rows, device=DEV)
        table = lambda *s: torch.zeros(*s, dtype=i32, device=DEV)
        angles = lambda *s: torch.ones(*s, device=DEV)
        step = lambda t: pkg.kv_step(ctx, ones, rows, pos, pool, ring, t)
        attend = lambda t: pkg.kv_attend(ctx, q, cache, t, ones, off, pos, scale=1.0, max_q=1, max_kv=1)
        store = lambda c, rot: pkg.kv_store(ctx, q, k, k, pos, slot, cache, c, rot_dim=rot)
        for way in (ctx._bind, None):
            monkeypatch.setattr(ctx, "_bind", way)
            for call in (step, attend):
                for bad in (table(rows, width + 1), table(2 * rows, width - 1), table(rows, 2 * width), table(1, rows * width), table(rows, width, 2)):
                    with pytest.raises(ValueError):
                        call(bad)
                    assert not bad.any()
                for good in (table(rows, width), table(rows + 2, width), table(rows * width), table(rows, 2, width // 2)):
                    call(good)
            for bad, rot in ((angles(9, d), d // 2), (angles(9, d // 2), d), (angles(9, 2, d), d), (angles(40, 16), 32)):
                cache.fill_(7)
                with pytest.raises(ValueError):
                    store(bad, rot)
                assert (cache == 7).all()
            for good, rot in ((angles(9, d), d), (angles(9, d // 2), d // 2), (angles(9, 2, d // 2), d), (angles(9, d), 0), (None, 0)):
                store(good, rot)
        for bad in (table(rows, width + 1), table(2 * rows, width - 1)):
            with pytest.raises(ValueError):
                ctx.wf_kv_attend(q, rows, cache, bad, ones, off, pos, rows, 1.0, torch.empty_like(q))
        with pytest.raises(ValueError):
            ctx.wf_kv_store(q, k, k, rows, pos, slot, torch.empty_like(q), cache, cos_sin=angles(9, d), n_pos=9, rot_dim=d // 2)
        torch.cuda.synchronize()


def test_other_threads_run_during_a_call():
    """A call that waits in the library (here: one that only sleeps) does not stop the interpreter's other threads."""
    import ctypes
    import threading
    with ctx_of(4, 2, 64, 16, 8, 4) as ctx:
        assert ctx._bind is not None, "_kvbind is not built"
        address = lambda f: ctypes.cast(f, ctypes.c_void_p).value
        lib = ctx.lib
        calls = [address(f) for f in (lib.wf_kv_step, lib.wf_kv_store, lib.wf_kv_load, lib.wf_kv_attend)]
        microseconds = 300000                                   # usleep's argument, in the context's place
        asleep = ctx._bind.geometry(microseconds, 0, 4, 2, 64, 8, 4, ctx.cache_bytes, False)
        cache, slot = torch.zeros(ctx.cache_bytes, dtype=torch.uint8, device=DEV), torch.arange(3, device=DEV)
        ticks, done = [], threading.Event()

        def other():
            while not done.wait(0.01):
                ticks.append(1)
        thread = threading.Thread(target=other)
        thread.start()
        try:
            ctx._bind.calls(calls[0], calls[1], address(ctypes.CDLL(None).usleep), calls[3])
            before = len(ticks)
            out = ctx._bind.load(asleep, 0, cache, slot)
            during = len(ticks) - before
        finally:
            ctx._bind.calls(*calls)
            done.set()
            thread.join()
        assert isinstance(out, tuple) and during >= 5, during


@pytest.mark.parametrize("n", [1000, 9000])
def test_attend_on_several_streams_at_once(n):
    """Rows in shares, joined by the last workgroup (1,000 tokens) or by a launch of their own, on two streams whose
    calls overlap: the results of each alone.  Streams past those with a work area: right too."""
    hq, hk, d, b = 8, 2, 128, 16
    rng = np.random.default_rng(n)
    q, cache, table, kv, q_off, pos = attend_case(rng, hq, hk, d, b, [(n, 1, None), (n // 2 + 3, 1, None)], "bf16")
    want, mag, dots = K.attend(host(q), cache, table, kv, q_off, pos, d ** -0.5, 0)
    with ctx_of(hq, hk, d, b, cache.n, table.shape[1]) as ctx:
        c, tb, ln, qo, ps = dev(cache.bytes), dev(table), dev(kv), dev(q_off), dev(pos)
        run = lambda x, **kw: pkg.kv_attend(ctx, x, c, tb, ln, qo, ps, scale=d ** -0.5, max_q=1, max_kv=n, **kw)
        inputs = [q, torch.roll(q, 1, 1)]
        alone = [run(x) for x in inputs]
        torch.cuda.synchronize()
        streams = [torch.cuda.Stream() for _ in range(12)]
        outs = [[], []]
        for _ in range(300):
            for x, s, out in zip(inputs, streams, outs):
                out.append(run(x, stream=s))
        torch.cuda.synchronize()
        for out, w in zip(outs, alone):
            for o in out:
                assert torch.equal(o, w)
        every = [run(q, stream=s) for s in streams]
        torch.cuda.synchronize()
        lim = bound("bf16", want, mag, dots, d, n)
        for o in every:
            assert (np.abs(host(o) - want) <= lim).all()
        assert torch.equal(every[0], alone[0]) and torch.equal(run(q), alone[0])


def test_arrays_of_the_host_are_a_type_error():
    """numpy arrays where device tensors belong, those with rows too."""
    with ctx_of(4, 2, 64, 16, 32, 4) as ctx:
        i32 = torch.int32
        q, k = torch.ones(3, 4, 64, dtype=torch.bfloat16, device=DEV), torch.ones(3, 2, 64, dtype=torch.bfloat16, device=DEV)
        cache = torch.zeros(ctx.cache_bytes, dtype=torch.uint8, device=DEV)
        ones, off, slot = torch.ones(3, dtype=i32, device=DEV), torch.arange(4, dtype=i32, device=DEV), torch.arange(3, device=DEV)
        table = torch.zeros(3, 4, dtype=i32, device=DEV)
        for bad in (dict(table=np.zeros((3, 4), np.int32)), dict(lens=np.ones(3, np.int32))):
            a = {**dict(table=table, lens=ones), **bad}
            with pytest.raises(TypeError):
                pkg.kv_attend(ctx, q, cache, a["table"], a["lens"], off, ones - 1, scale=1.0)
        with pytest.raises(TypeError):
            pkg.kv_store(ctx, q, k, k, ones, slot, cache, np.ones((9, 64), np.float32), rot_dim=64)
