"""The 8-bit cache on the GPU against the oracle of kv8_oracle.py: norm + rotation + store, load, attention."""
import numpy as np
import pytest
import torch

import kv8_oracle as E
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
    return pkg.KVContext(0, q_heads=hq, kv_heads=hk, head_dim=d, block_tokens=b, n_blocks=n, max_blocks=width, dtype=dtype, codes="e4m3")


def dev(x, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(x)).to(DEV)
    return t if dtype is None else t.to(dtype)


def host(t):
    return t.float().cpu().numpy()


def filled(rng, n, hk, b, d):
    """A cache of any finite codes, with scales of different sizes."""
    c = E.Cache8(n, hk, b, d, rng)
    codes = c.bytes[..., :2 * b * d]
    codes[(codes & 0x7f) == 0x7f] = 0x33
    for blk in range(n):
        for h in range(hk):
            for i in range(2):
                c.put_scale(blk, h, i, int(rng.integers(-10, -6)))
    return c


# ---- store and load ----------------------------------------------------------------------------

def runs_of_slots(rng, T, b, longest, whole=False):
    """Slots of T tokens as steps give them: rows of consecutive tokens, from anywhere in a block, in blocks of any order; a
    row without slots now and then.  And the number of blocks."""
    slot, used = [], 0
    while len(slot) < T:
        n, first = int(rng.integers(1, longest + 1)), 0 if whole else int(rng.integers(0, b))
        n = min(n, T - len(slot))
        if rng.random() < 0.1:
            slot += [-1] * n
        else:
            slot += [used * b + first + i for i in range(n)]
            used += -(-(first + n) // b)
    order = rng.permutation(max(used, 1))
    slot = np.array(slot)
    return np.where(slot < 0, -1, order[np.maximum(slot, 0) // b] * b + slot % b).astype(np.int64), max(used, 1)


def store_case(rng, hq, hk, d, T, dtype, rot, pad=0, scale=1.0):
    width = (hq + 2 * hk) * d + pad
    # heads and tokens of different sizes, so that scales rise and stay
    x = rng.standard_normal((T, width)) * np.exp(rng.standard_normal((T, 1))) * scale
    qkv = dev(x.astype(np.float32), TYPES[dtype])
    part = lambda a, n: qkv[:, a * d:(a + n) * d].unflatten(-1, (n, d))
    n_pos = 977
    angle = np.arange(n_pos)[:, None] * 1e4 ** (-np.arange(0, max(rot, 2), 2) / max(rot, 2))
    cs = np.concatenate([np.cos(angle), np.sin(angle)], 1).astype(np.float32)
    return part(0, hq), part(hq, hk), part(hq + hk, hk), rng.integers(0, n_pos, T).astype(np.int32), cs


SHAPES = [(4, 2, 64), (5, 1, 128), (2, 2, 256)]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("hq,hk,d", SHAPES)
@pytest.mark.parametrize("b", [16, 32, 64, 128, 256])
def test_store_bytes(hq, hk, d, b, dtype):
    """Without norm and rotation the cache is the oracle's to the last bit, in blocks that begin, go on under a scale
    that holds, and go on under one that rises."""
    rng = np.random.default_rng(d + b)
    for T, longest in ((1, 1), (37, 1), (60, 9), (300, 2 * b), (2 * b + 5, 4 * b)):
        q, k, v, pos, _ = store_case(rng, hq, hk, d, T, dtype, 0, pad=8)
        slot, n = runs_of_slots(rng, T, b, longest)
        want = filled(rng, n + 1, hk, b, d)
        cache = dev(want.bytes)
        want.put(slot, host(k), host(v))
        with ctx_of(hq, hk, d, b, n + 1, 4, dtype) as ctx:
            out = pkg.kv_store(ctx, q, k, v, None, dev(slot), cache)
            assert torch.equal(out, q)
            assert np.array_equal(cache.cpu().numpy(), want.bytes), (T, longest)
            # what is loaded is what the oracle holds, rounded, at most the type's largest
            lk, lv = pkg.kv_load(ctx, cache, dev(slot))
            top = torch.finfo(TYPES[dtype]).max
            for x, y in zip((lk, lv), want.get(np.maximum(slot, 0))):
                y[slot < 0] = 0
                assert torch.equal(x.cpu(), torch.from_numpy(y.clip(-top, top)).to(TYPES[dtype]))
            # once more: nothing changes (scales hold, or begin with the same tokens)
            again = cache.clone()
            pkg.kv_store(ctx, q, k, v, None, dev(slot), again)
            assert torch.equal(again, cache)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("hq,hk,d", SHAPES)
def test_store_norm_and_rotation(hq, hk, d, dtype):
    for i, (T, b, rot, inter, norm) in enumerate([(1, 16, d, False, True), (33, 32, d // 2, True, True), (70, 64, 16, False, False),
                                                  (5, 16, 0, False, True), (129, 128, d, True, False), (40, 256, d // 4, False, True)]):
        rng = np.random.default_rng(i)
        q, k, v, pos, cs = store_case(rng, hq, hk, d, T, dtype, rot, pad=8 * (i % 3))
        wq, wk = (dev((1 + 0.2 * rng.standard_normal(d)).astype(np.float32), TYPES[dtype]) for _ in range(2))
        slot, n = runs_of_slots(rng, T, b, b, whole=True)
        if T == 1:
            slot, n = np.array([0]), 1
        got = E.Cache8(n, hk, b, d)
        with ctx_of(hq, hk, d, b, n, 4, dtype) as ctx:
            cache = dev(got.bytes)
            out = pkg.kv_store(ctx, q, k, v, dev(pos), dev(slot), cache, dev(cs) if rot else None, rot_dim=rot, interleaved=inter,
                               q_weight=wq if norm else None, k_weight=wk if norm else None, eps=1e-5)
            got.bytes = cache.cpu().numpy()
        u, tiny = UNIT[dtype], 2.0 ** -25 if dtype == "f16" else 2.0 ** -134
        want = K.normed_rotated(host(q), host(wq) if norm else None, 1e-5, cs, pos, rot, inter)
        size = np.abs(want).max(-1, keepdims=True) * 2 + 1e-30
        # one rounding to 16 bits, and fp32 roundings of the norm (its sum's, halved by the root) and the rotation
        assert (np.abs(host(out) - want) <= u * np.abs(want) + 16 * 2.0 ** -24 * size + tiny).all()
        live = slot >= 0
        want = K.normed_rotated(host(k), host(wk) if norm else None, 1e-5, cs, pos, rot, inter)[live]
        blk, off = slot[live] // b, slot[live] % b
        # a block's scale is that of its largest magnitude (fp32 may take one at a border for the next)
        s = got.scales()[blk, :, 0].astype(np.float64)
        for x in np.unique(blk):
            for h in range(hk):
                most = np.abs(want[blk == x, h]).max()
                near = {E.least_power(most * (1 + e)) for e in (-1e-5, 0, 1e-5)}
                assert int(np.log2(got.scales()[x, h, 0])) in near
        # the nearest code, or the other one where fp32's value may be on the other side of half-way
        c = got.keys()[blk, :, off]
        fit = np.zeros(c.shape, bool)
        for e in (-1, 0, 1):
            move = e * 40 * 2.0 ** -24 * np.abs(want).max(-1, keepdims=True)
            fit |= c == E.codes((want + move) / s[..., None])
        # (a zero may have either sign)
        assert (fit | ((c & 0x7f) == 0) & (np.abs(want) <= 2.0 ** -10 * s[..., None] * (1 + 1e-5))).all()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_store_every_value(dtype):
    """Every 16-bit value beside ones that set the scale: largest, smallest, zeros, infinities, NaN, as the oracle."""
    d, b, hk = 64, 16, 1
    bits = np.arange(1 << 16, dtype=np.uint32).astype(np.uint16)
    x = torch.from_numpy(bits.view(np.int16)).view(TYPES[dtype])
    T = (1 << 16) // d
    k = x.view(T, 1, d)
    v = x[torch.from_numpy(np.random.default_rng(3).permutation(1 << 16))].view(T, 1, d)
    with np.errstate(all="ignore"):
        for order in (np.arange(T), np.random.default_rng(0).permutation(T)):
            kk, vv = k[order], v[order]
            if order[0] != 0:      # finite ones alone, in blocks of one size: no token is dropped as a whole
                ok = torch.isfinite(x.float())
                f = x[ok][:ok.sum() // d * d]
                kk = f.view(-1, 1, d)
                vv = f.flip(0).contiguous().view(-1, 1, d)
            t = len(kk)
            slot = np.arange(t, dtype=np.int64)
            n = -(-t // b)
            want = E.Cache8(n, hk, b, d)
            want.put(slot, kk.float().numpy(), vv.float().numpy())
            cache = torch.zeros(want.bytes.size, dtype=torch.uint8, device=DEV)
            with ctx_of(1, 1, d, b, n, 4, dtype) as ctx:
                pkg.kv_store(ctx, kk.to(DEV), kk.to(DEV), vv.to(DEV), None, dev(slot), cache)
                got = cache.cpu().numpy().reshape(want.bytes.shape)
                assert np.array_equal(got, want.bytes)
                lk, lv = pkg.kv_load(ctx, cache, dev(slot))
            top = torch.finfo(TYPES[dtype]).max
            for a, w in zip((lk, lv), want.get(slot)):
                w = torch.from_numpy(w.clip(-top, top)).to(TYPES[dtype])
                assert torch.equal(a.cpu().isnan(), w.isnan()) and torch.equal(a.cpu().nan_to_num(), w.nan_to_num())


def test_store_ranges_of_scales():
    """Scales from the least to the largest, and codes rounded from each to the next: as the oracle."""
    d, b = 64, 16
    rng = np.random.default_rng(5)
    x = rng.standard_normal((b, 2, 1, d)).astype(np.float32)
    want = E.Cache8(1, 1, b, d)
    cache = dev(want.bytes)
    # every token far above the one before; the first ones vanish
    size = 2.0 ** np.array([-126, -120, -115, -110, -100, -95, -90, -60, -20, 0, 5, 40, 100, 120, 126, 126.9])
    k = torch.from_numpy((x[:, 0] * size[:, None, None]).astype(np.float32)).clamp(-3e38, 3e38).to(torch.bfloat16)
    v = torch.from_numpy((x[:, 1] * size[:, None, None]).astype(np.float32)).clamp(-3e38, 3e38).to(torch.bfloat16)
    with ctx_of(1, 1, d, b, 1, 1) as ctx:
        for t in range(b):
            pkg.kv_store(ctx, k[t:t + 1].to(DEV), k[t:t + 1].to(DEV), v[t:t + 1].to(DEV), None, dev(np.array([t])), cache)
            want.put([t], k[t:t + 1].float().numpy(), v[t:t + 1].float().numpy())
            assert np.array_equal(cache.cpu().numpy().reshape(-1), want.bytes.reshape(-1)), t


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("hq,hk,d,b,longest", [(12, 4, 64, 16, 300), (14, 1, 128, 32, 40), (9, 3, 256, 64, 700), (16, 2, 128, 16, 3)])
def test_store_many_tokens(hq, hk, d, b, longest, dtype):
    """Large calls: the same bytes and queries as the tokens of a few blocks at a time."""
    rng = np.random.default_rng(d + b)
    T = 40000 // hq + 13
    q, k, v, pos, cs = store_case(rng, hq, hk, d, T, dtype, d, pad=8)
    slot, n = runs_of_slots(rng, T, b, longest)
    w = dev((1 + 0.2 * rng.standard_normal(d)).astype(np.float32), TYPES[dtype])
    p, sl, c = dev(pos), dev(slot), dev(cs)
    blk = np.where(slot < 0, -1, slot // b)
    cuts = [0]
    for t in range(1, T):
        if blk[t] != blk[t - 1] and t - cuts[-1] > 300:
            cuts.append(t)
    before = dev(filled(rng, n, hk, b, d).bytes).view(-1)
    with ctx_of(hq, hk, d, b, n, 4, dtype) as ctx:
        for how in (dict(rot_dim=d, q_weight=w, k_weight=w), dict(rot_dim=d // 2, k_weight=w), dict(rot_dim=d // 4, interleaved=True), dict()):
            table = (c[:, :how["rot_dim"]].contiguous(),) if how.get("rot_dim") else ()
            one, parts = before.clone(), before.clone()
            out = pkg.kv_store(ctx, q, k, v, p, sl, one, *table, **how)
            for t, e in zip(cuts, cuts[1:] + [T]):
                got = pkg.kv_store(ctx, q[t:e], k[t:e], v[t:e], p[t:e].clone(), sl[t:e].clone(), parts, *table, **how)
                assert torch.equal(got, out[t:e]), (how, t)
            assert torch.equal(one, parts), how


def test_store_leaves_the_rest():
    """Nothing outside the blocks of the call's tokens changes, whatever the slots hold; a token without a slot
    between two of one block parts them."""
    d, b, hk, n = 64, 16, 2, 9
    rng = np.random.default_rng(6)
    q, k, v, pos, _ = store_case(rng, 4, hk, d, 12, "bf16", 0)
    slot = np.array([35, 36, -1, 2 ** 62, -2 ** 63, n * b, 37, 70, 71, 72, 2 ** 31, 100], np.int64)
    want = filled(rng, n, hk, b, d)
    guard = torch.full((want.bytes.size + 512,), 99, dtype=torch.uint8, device=DEV)
    cache = guard[256:-256]
    cache.copy_(dev(want.bytes).view(-1))
    with ctx_of(4, hk, d, b, n, 4) as ctx:
        # (35 and 36, then 37 by itself: a call each for the oracle, and so for the GPU)
        for part in (slice(0, 6), slice(6, 12)):
            pkg.kv_store(ctx, q[part], k[part], v[part], None, dev(slot[part]), cache)
            want.put(slot[part], host(k[part]), host(v[part]))
    assert np.array_equal(cache.cpu().numpy(), want.bytes.reshape(-1))
    assert (guard[:256] == 99).all() and (guard[-256:] == 99).all()


# ---- attention ---------------------------------------------------------------------------------

def attend_case(rng, hq, hk, d, b, rows, dtype, extra=2):
    """rows: (cached, queries, first position or None)."""
    kv = np.array([r[0] for r in rows])
    width = max(1, int((-(-kv // b)).max()))
    n = int((-(-kv // b)).sum()) + extra
    cache = filled(rng, n, hk, b, d)
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


def bound(dtype, want, mag, dots, d, n, top):
    """|error| of an output: its rounding, that of p (f16: of p times scale, relative u or half the type's smallest step, which
    is 2^-27 of the largest such term `top` at most, times a code), fp32 products and sums (n terms and the exponentials'), and the error
    of the scores, which multiplies p by at most 1 + 2 delta."""
    u = UNIT[dtype]
    tiny = 448 * n * 2.0 ** -27 * top[..., None] if dtype == "f16" else 0.0
    delta = (d + 16) * 2.0 ** -24 * dots[..., None]
    return u * np.abs(want) + (u * 1.01 + 2.2 * delta + (n + 64) * 2.0 ** -23) * mag + tiny + 2.0 ** -25


def check_attend(hq, hk, d, b, rows, dtype="bf16", window=0, seed=0, scale=None, hints=True, pad=0):
    rng = np.random.default_rng(seed)
    q, cache, table, kv, q_off, pos = attend_case(rng, hq, hk, d, b, rows, dtype)
    scale = 0.2 * d ** -0.5 if scale is None else scale
    want, mag, dots, top = E.attend(host(q), cache, table, kv, q_off, pos, scale, window)
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
            lim = bound(dtype, want, mag, dots, d, max(1, int(kv.max())), top)
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


@pytest.mark.parametrize("hq,hk,d,dtype", [(4, 1, 128, "bf16"), (8, 2, 64, "f16"), (6, 3, 256, "bf16"), (7, 1, 64, "bf16"), (4, 2, 256, "f16"),
                                           (8, 1, 128, "f16")])
def test_attend_long_prompts(hq, hk, d, dtype):
    """Several tiles of columns a row and many steps of tokens, with and without a window."""
    rows = [(700, 700, None), (390, 130, None), (64, 64, None), (0, 5, 0), (1000, 90, None)]
    check_attend(hq, hk, d, 32, rows, dtype, seed=d + hq)
    check_attend(hq, hk, d, 16, rows, dtype, seed=d + hq, window=150, hints=False)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("window", [0, 70])
def test_attend_many_columns_of_64_channels(window, dtype):
    """Enough columns in all for the kernel of many columns, which 64 channels take late."""
    rows = [(150, 150, None), (90, 30, None), (0, 5, 0), (300, 20, None), (40, 10, 35), (64, 3, -1)]
    check_attend(1024, 64, 64, 16, rows, dtype, seed=5, window=window, hints=False)


@pytest.mark.parametrize("window", [1, 2, 16, 63, 64, 100, 5000])
def test_attend_window(window):
    check_attend(8, 2, 64, 16, [(300, 1, None), (150, 90, None), (40, 40, None), (1, 1, None)], window=window, seed=window)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("window", [1, 16, 63, 100])
def test_attend_prompts_through_small_windows(window, dtype):
    check_attend(4, 1, 64, 16, [(600, 600, None), (300, 90, None)], dtype, window=window, seed=window)


def test_attend_empty_rows():
    """Rows without cached tokens (refused), positions before the first token and
    past the last, rows without queries."""
    rows = [(0, 3, 0), (5, 9, -4), (50, 0, None), (20, 4, 18), (0, 0, 0), (33, 5, 60), (7, 1, -1)]
    check_attend(8, 2, 128, 16, rows, window=0, seed=1)
    check_attend(8, 2, 128, 16, [(20, 6, 18), (33, 5, 60), (40, 3, -1)], window=4, seed=2)
    check_attend(8, 1, 64, 16, [(300, 80, -40), (40, 70, 20), (0, 90, 0), (200, 66, 500)], "f16", window=90, seed=3)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_attend_longer(dtype):
    check_attend(8, 2, 128, 64, [(5000, 1, None), (1100, 1, None), (3, 1, None)], dtype, seed=7)
    check_attend(4, 1, 64, 16, [(2100, 17, None), (900, 1, None)], dtype, seed=8)


def test_attend_large_scores():
    # one token takes nearly all the weight; negative and zero scales
    for scale in (1.0, -0.3, 0.0):
        check_attend(8, 2, 64, 16, [(500, 1, None), (60, 20, None)], scale=scale, seed=3)


def test_attend_strided_queries():
    check_attend(8, 2, 64, 16, [(90, 1, None), (60, 5, None)], pad=24, seed=4, hints=False)


def test_attend_many_rows():
    rng = np.random.default_rng(9)
    check_attend(4, 2, 64, 16, [(int(n), 1, None) for n in rng.integers(0, 90, 300)], seed=9)


@pytest.mark.parametrize("hq,hk,d,nq", [(8, 1, 64, 3), (8, 1, 128, 16), (16, 1, 128, 20), (4, 1, 256, 90)])
def test_attend_few_queries_over_many_tokens(hq, hk, d, nq):
    check_attend(hq, hk, d, 32, [(3000, nq, None)], seed=nq)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("nq", [3, 6, 7, 16])
def test_attend_256_channels_between_single_tokens_and_prompts(nq, dtype):
    check_attend(8, 1, 256, 16, [(2900, nq, None), (70, nq, None), (nq, nq, None), (0, 0, None)], dtype, seed=nq)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("hq,hk,d,nq", [(8, 1, 64, 1), (8, 2, 128, 1), (8, 1, 64, 30), (4, 1, 128, 200), (1024, 16, 64, 50)])
@pytest.mark.parametrize("scale", [-0.05, 0.0])
def test_attend_scales_that_are_not_positive(scale, hq, hk, d, nq, dtype):
    check_attend(hq, hk, d, 16, [(210, nq, None), (33, min(nq, 33), None)], dtype, scale=scale, seed=nq, hints=False)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("hq,hk,d,nq", [(8, 1, 64, 1), (8, 1, 64, 30), (4, 1, 128, 200), (4, 1, 256, 40)])
def test_attend_blocks_of_zeros(hq, hk, d, nq, dtype):
    """Blocks whose values are all 0 have the least scale: their probabilities count in the total all the same."""
    rng = np.random.default_rng(nq)
    b, n = 16, 304
    q, cache, table, kv, q_off, pos = attend_case(rng, hq, hk, d, b, [(n, nq, None)], dtype)
    T = n
    x = rng.standard_normal((2, T, hk, d)).astype(np.float32)
    x[1, (np.arange(T) // b) % 3 > 0] = 0
    slot = table[0, np.arange(T) // b].astype(np.int64) * b + np.arange(T) % b
    with ctx_of(hq, hk, d, b, cache.n, table.shape[1], dtype) as ctx:
        raw = dev(cache.bytes).view(-1)
        k, v = dev(x[0], TYPES[dtype]), dev(x[1], TYPES[dtype])
        pkg.kv_store(ctx, torch.zeros(T, hq, d, dtype=TYPES[dtype], device=DEV), k, v, dev(np.arange(T, dtype=np.int32)), dev(slot), raw)
        cache.bytes = raw.cpu().numpy().reshape(cache.bytes.shape)
        want, mag, dots, top = E.attend(host(q), cache, table, kv, q_off, pos, 0.1, 0)
        got = host(pkg.kv_attend(ctx, q, raw, dev(table), dev(kv), dev(q_off), dev(pos), scale=0.1, max_q=nq, max_kv=n))
    assert (np.abs(got - want) <= bound(dtype, want, mag, dots, d, n, top)).all()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("hq,hk,d,b,nq,window", [(8, 2, 64, 16, 1, 50), (8, 2, 64, 16, 13, 50), (8, 2, 128, 32, 1, 0), (4, 1, 256, 16, 40, 33),
                                                 (8, 1, 64, 16, 150, 60), (4, 1, 128, 64, 150, 0), (4, 1, 256, 32, 150, 20),
                                                 (1024, 16, 64, 16, 110, 60)])
def test_attend_beside_garbage(hq, hk, d, b, nq, window, dtype):
    """Codes and scales that are no numbers, past a row's end, before its window, and in blocks of no row (as freed or never used
    memory has); ids of unused table entries out of range."""
    rng = np.random.default_rng(11)
    rows = [(37, min(nq, 37), None), (100, min(nq, 100), None), (290, nq, None), (0, 1, 0)]
    q, cache, table, kv, q_off, pos = attend_case(rng, hq, hk, d, b, rows, dtype)
    scale = 0.2 * d ** -0.5
    want, mag, dots, top = E.attend(host(q), cache, table, kv, q_off, pos, scale, window)
    seen = np.zeros((cache.n, b), bool)
    for r, (n, m, _) in enumerate(rows):
        for j in range(max(0, n - m - window + 1) if window else 0, n):
            seen[table[r, j // b], j % b] = True
    vc = cache.value_codes()
    for blk in range(cache.n):
        for h in range(hk):
            cache.keys()[blk, h][~seen[blk]] = 0x7f
            vc[blk, h][~seen[blk]] = 0xff
            cache.put_values(blk, h, vc[blk, h])
            if not seen[blk].any():
                cache.bytes[blk, h, 2 * b * d:2 * b * d + 8] = np.array([np.nan, rng.choice([np.nan, np.inf, -np.inf])], np.float32).view(np.uint8)
    keys = cache.keys().copy()
    keys[~np.broadcast_to(seen[:, None], keys.shape[:3])] = 0x7f
    cache.bytes[..., :b * d] = keys.reshape(cache.n, hk, -1)
    table = np.where(table < 0, rng.choice(np.array([-1, 2 ** 31 - 1, -2 ** 31, cache.n], np.int32), table.shape), table).astype(np.int32)
    with ctx_of(hq, hk, d, b, cache.n, table.shape[1], dtype) as ctx:
        for max_kv in (290, 0):   # (unknown: the kernel of many columns where there are any)
            got = host(pkg.kv_attend(ctx, q, dev(cache.bytes), dev(table), dev(kv), dev(q_off), dev(pos), scale=scale, window=window,
                                     max_q=nq, max_kv=max_kv))
            assert (np.abs(got - want) <= bound(dtype, want, mag, dots, d, 290, top)).all()


@pytest.mark.parametrize("what", ["key", "value"])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("nq,hq,d", [(40, 4, 64), (200, 4, 128), (110, 1024, 64 * 2), (200, 1024, 64)])
def test_a_token_that_is_no_number_shows_where_it_is_seen(what, nq, hq, d, dtype):
    """Stored with a NaN or an infinity, it reaches the queries that see it, and no others."""
    hk, b = 2, 16
    rng = np.random.default_rng(12)
    q, k, v, pos, _ = store_case(rng, hq, hk, d, nq, dtype, 0)
    (k if what == "key" else v)[20, 1, 5] = np.inf if what == "key" else np.nan
    n = -(-nq // b)
    with ctx_of(hq, hk, d, b, n, n, dtype) as ctx:
        cache = torch.full((ctx.cache_bytes,), 255, dtype=torch.uint8, device=DEV)
        slot, i32 = torch.arange(nq, device=DEV), torch.int32
        pkg.kv_store(ctx, q, k, v, None, slot, cache)
        lk, lv = pkg.kv_load(ctx, cache, slot)
        for x in (lk, lv):
            assert x[20, 1].isnan().all() and x[20, 0].isfinite().all() and x[:20].isfinite().all() and x[21:].isfinite().all()
        out = pkg.kv_attend(ctx, q, cache, torch.arange(n, dtype=i32, device=DEV)[None], dev(np.array([nq], np.int32)),
                            dev(np.array([0, nq], np.int32)), slot.to(i32), scale=0.125, max_q=nq)
    assert out[20:, hq // 2:].isnan().all() and out[:20].isfinite().all() and out[:, :hq // 2].isfinite().all()


def skewed_case(rng, hq, hk, d, b, n, nq, dtype, far, size=1.0):
    """nq queries of one row over n tokens; the blocks in `far` have large keys along the queries' direction and values `size` as large."""
    q, cache, table, kv, q_off, pos = attend_case(rng, hq, hk, d, b, [(n, nq, None)], dtype)
    base = rng.standard_normal((hk, 1, d))
    x = np.repeat(base, hq // hk, axis=1).reshape(hq, d) + 0.3 * rng.standard_normal((nq, hq, d))
    for j in far:
        blk = table[0, j // b]
        for h in range(hk):
            k = np.zeros((b, d)) + base[h] * 3
            e = E.least_power(np.abs(k).max())
            cache.bytes[blk, h, :b * d] = E.codes(k / 2.0 ** e).reshape(-1)
            cache.put_scale(blk, h, 0, e)
            cache.put_scale(blk, h, 1, int(np.log2(size)) - 7)
    return dev(x.astype(np.float32), TYPES[dtype]), cache, table, kv, q_off, pos


@pytest.mark.parametrize("size", [1.0, 2.0 ** -12, 2.0 ** 12])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("hq,hk,d,nq", [(8, 1, 64, 1), (8, 1, 64, 200), (4, 1, 128, 150), (6, 1, 256, 100), (984, 8, 64, 200)])
def test_attend_uneven_scores_and_values(hq, hk, d, nq, dtype, size):
    """Blocks that take nearly all the weight, early, late or in the middle, with values far smaller or larger than the others'."""
    n, b = 1500, 16
    for i, far in enumerate(([0], [700], [1499 - nq // 2], [40, 900, 1400])):
        if hq > 100 and i in (1, 2):      # (many heads: half of them)
            continue
        rng = np.random.default_rng(100 + i)
        q, cache, table, kv, q_off, pos = skewed_case(rng, hq, hk, d, b, n, nq, dtype, far, size)
        scale = 0.5 * d ** -0.5
        want, mag, dots, top = E.attend(host(q), cache, table, kv, q_off, pos, scale, 0)
        with ctx_of(hq, hk, d, b, cache.n, table.shape[1], dtype) as ctx:
            for max_kv in (n, 0):
                got = host(pkg.kv_attend(ctx, q, dev(cache.bytes), dev(table), dev(kv), dev(q_off), dev(pos), scale=scale, max_q=nq,
                                         max_kv=max_kv))
                lim = bound(dtype, want, mag, dots, d, n, top)
                assert (np.abs(got - want) <= lim).all(), (far, max_kv, float((np.abs(got - want) / lim).max()))


def test_attend_large_positions_and_windows():
    """Positions past every window and at the ends of 32 bits."""
    rng = np.random.default_rng(21)
    for nq in (1, 40):
        q, cache, table, kv, q_off, pos = attend_case(rng, 8, 2, 64, 16, [(100, nq, None), (60, nq, None)], "bf16")
        for window in (1, 64, 2 ** 31 - 1):
            for p in (2 ** 31 - 1, 2 ** 31 - 64, 99 + window if window < 2 ** 30 else 99, -2 ** 31, 160):
                pos[:] = min(p, 2 ** 31 - 1)
                want, mag, dots, top = E.attend(host(q), cache, table, kv, q_off, pos.astype(np.int64), 0.05, window)
                with ctx_of(8, 2, 64, 16, cache.n, table.shape[1]) as ctx:
                    got = host(pkg.kv_attend(ctx, q, dev(cache.bytes), dev(table), dev(kv), dev(q_off), dev(pos), scale=0.05,
                                             window=window, max_q=nq, max_kv=100))
                assert (np.abs(got - want) <= bound("bf16", want, mag, dots, 64, 100, top)).all(), (nq, window, p)


def test_attend_cache_past_32_bits():
    """Blocks whose bytes are past 2^32, and rows behind the last query left as they were."""
    hq, hk, d, b = 4, 2, 128, 256
    n = (1 << 32) // (hk * (2 * b * d + 16)) + 40
    rng = np.random.default_rng(13)
    with ctx_of(hq, hk, d, b, n, 3) as ctx:
        cache = torch.zeros(ctx.cache_bytes, dtype=torch.uint8, device=DEV)
        blocks = np.array([[n - 1, 3, n - 30], [n - 7, n - 2, 0]])
        T = 600
        q, k, v, pos, _ = store_case(rng, hq, hk, d, 2 * T, "bf16", 0)
        at = np.arange(T)
        slot = np.concatenate([blocks[r][at // b] * b + at % b for r in range(2)])
        pkg.kv_store(ctx, q, k, v, None, dev(slot), cache)
        small = E.Cache8(6, hk, b, d)
        mine = {x: i for i, x in enumerate(blocks.reshape(-1))}
        small.put(np.array([mine[s // b] * b + s % b for s in slot]), host(k), host(v))
        lk, lv = pkg.kv_load(ctx, cache, dev(slot))
        wk, wv = small.get(np.array([mine[s // b] * b + s % b for s in slot]))
        assert np.array_equal(host(lk), wk) and np.array_equal(host(lv), wv)
        qq = torch.cat([q[T - 1:T], q[2 * T - 1:]])
        pad = torch.cat([qq, qq, qq])
        out = torch.full_like(pad, 7.0)
        kv, off, p = (dev(np.array(x, np.int32)) for x in ([T, T], [0, 1, 2], [T - 1] * 6))
        table = dev(blocks.astype(np.int32))
        ctx.wf_kv_attend(pad, 6, cache, table, kv, off, p, 2, 0.1, out, max_q=1, max_kv=T)
        want, mag, dots, top = E.attend(host(qq), small, np.arange(6).reshape(2, 3), [T, T], [0, 1, 2], [T - 1] * 2, 0.1, 0)
        assert (np.abs(host(out[:2]) - want) <= bound("bf16", want, mag, dots, d, T, top)).all()
        assert (out[2:] == 7).all()


# ---- streams, graphs, refusals -----------------------------------------------------------------

@pytest.mark.parametrize("prompt", [1, 90])
def test_a_whole_step_replays(prompt):
    """Step, store, attention and load from one graph, several times, with the program's own work between: as eager calls."""
    hq, hk, d, b, n, rows = 8, 2, 64, 16, 200, 3
    rng = np.random.default_rng(31)
    T = prompt * rows
    q, k, v, _, cs = store_case(rng, hq, hk, d, T, "bf16", d)
    with ctx_of(hq, hk, d, b, n, 60) as ctx:
        new = torch.full((rows,), prompt, dtype=torch.int32, device=DEV)
        start = (dev(np.array([5, 0, 31], np.int32)), torch.tensor([0, n - 8], dtype=torch.int32, device=DEV))
        ring = torch.arange(n, dtype=torch.int32, device=DEV)
        table = torch.full((rows, 60), -1, dtype=torch.int32, device=DEV)
        table[0, 0], table[2, 0], table[2, 1] = n - 1, n - 2, n - 3
        first = dev(filled(rng, n, hk, b, d).bytes).view(-1)
        cs = dev(cs)

        def step(lens, pool, ring, table, cache):
            lens, pool, off, slot, pos, _ = pkg.kv_step(ctx, new, T, lens, pool, ring, table)
            x = pkg.kv_store(ctx, q, k, v, pos, slot, cache, cs, rot_dim=d)
            out = pkg.kv_attend(ctx, x, cache, table, lens, off, pos, scale=0.1, max_q=prompt, max_kv=40 + prompt)
            return lens, pool, out, *pkg.kv_load(ctx, cache, slot)

        def eager(times):
            state = [x.clone() for x in start]
            r, t, c = ring.clone(), table.clone(), first.clone()
            for _ in range(times):
                lens, pool, *rest = step(*state, r, t, c)
                state = [lens, pool]
            return [lens, pool, *rest, c, t]

        lens, pool = (x.clone() for x in start)
        r, t, c = ring.clone(), table.clone(), first.clone()
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            step(lens, pool, r, t, c)                    # (warm)
            side.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                outs = step(lens, pool, r, t, c)
                lens.copy_(outs[0])
                pool.copy_(outs[1])
        for x, y in zip((lens, pool, r, t, c), (*start, ring, table, first)):
            x.copy_(y)
        for times in range(1, 5):
            graph.replay()
            torch.cuda.synchronize()
            want = eager(times)
            for x, y in zip([*outs, c, t], want):
                assert torch.equal(x, y), times


def test_calls_on_streams_at_once():
    """Attention of one context on several streams, on data of their own."""
    rng = np.random.default_rng(41)
    cases = [attend_case(rng, 8, 1, 64, 16, [(3000 + 64 * i, 1, None)], "bf16", extra=0) for i in range(3)]
    n, width = max(c[1].n for c in cases), max(c[2].shape[1] for c in cases)
    with ctx_of(8, 1, 64, 16, n, width) as ctx:
        sets = []
        for q, cache, table, kv, off, pos in cases:
            full = np.zeros((n, *cache.bytes.shape[1:]), np.uint8)
            full[:cache.n] = cache.bytes
            wide = np.full((1, width), -1, np.int32)
            wide[:, :table.shape[1]] = table
            sets.append((q, dev(full), dev(wide), dev(kv), dev(off), dev(pos)))
        call = lambda s: pkg.kv_attend(ctx, *s, scale=0.05, max_q=1, max_kv=4000)
        want = [call(s) for s in sets]
        streams = [torch.cuda.Stream() for _ in range(11)]
        torch.cuda.synchronize()
        got = []
        for i in range(33):
            with torch.cuda.stream(streams[i % 11]):
                got.append(call(sets[i % 3]))
        torch.cuda.synchronize()
        for i, x in enumerate(got):
            # (streams past the first eight do not share tokens out: sums in another order)
            assert torch.allclose(x.float(), want[i % 3].float(), rtol=2 ** -6, atol=2 ** -8 * float(want[i % 3].abs().max()))


def test_refusals():
    with ctx_of() as ctx:
        q = torch.zeros(4, 8, 64, dtype=torch.bfloat16, device=DEV)
        k = torch.zeros(4, 2, 64, dtype=torch.bfloat16, device=DEV)
        cache = torch.zeros(ctx.cache_bytes, dtype=torch.uint8, device=DEV)
        slot = torch.arange(4, device=DEV)
        with pytest.raises((ValueError, TypeError)):
            pkg.kv_store(ctx, q, k, k, None, slot, cache[:-1])
        with pytest.raises(TypeError):
            pkg.kv_store(ctx, q.half(), k, k, None, slot, cache)
        with pytest.raises(pkg.WFError):
            pkg.kv_store(ctx, q, k, k, slot.int(), slot, cache, rot_dim=64)
        with pytest.raises(pkg.WFError):
            pkg.kv_store(ctx, q, k, k, None, slot, cache, eps=-1.0)
        one = torch.zeros(2, dtype=torch.int32, device=DEV)
        for bad in (dict(scale=float("nan")), dict(scale=1.0, window=-1), dict(scale=1.0, max_kv=-1)):
            with pytest.raises(pkg.WFError):
                pkg.kv_attend(ctx, q, cache, torch.zeros(1, 8, dtype=torch.int32, device=DEV), one[:1], one, slot.int(), **bad)
    # a cache of 4-bit codes is smaller
    with pkg.KVContext(0, q_heads=8, kv_heads=2, head_dim=64, block_tokens=16, n_blocks=64, max_blocks=8) as four:
        with ctx_of() as ctx:
            assert four.cache_bytes < ctx.cache_bytes and four.codes == "e2m1" and ctx.codes == "e4m3"
            with pytest.raises((ValueError, TypeError)):
                pkg.kv_load(ctx, torch.zeros(four.cache_bytes, dtype=torch.uint8, device=DEV), torch.zeros(1, dtype=torch.int64, device=DEV))


def test_no_tokens():
    with ctx_of() as ctx:
        q = torch.zeros(0, 8, 64, dtype=torch.bfloat16, device=DEV)
        k = torch.zeros(0, 2, 64, dtype=torch.bfloat16, device=DEV)
        cache = torch.full((ctx.cache_bytes,), 5, dtype=torch.uint8, device=DEV)
        none = torch.zeros(0, dtype=torch.int64, device=DEV)
        assert pkg.kv_store(ctx, q, k, k, None, none, cache).shape == (0, 8, 64)
        assert pkg.kv_load(ctx, cache, none)[0].shape == (0, 2, 64)
        assert (cache == 5).all()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("window", [1, 40, 63, 64, 150, 333])
@pytest.mark.parametrize("hq,hk,d,b", [(8, 1, 128, 32), (10, 2, 128, 16), (6, 3, 256, 32)])
def test_attend_prompts_of_many_columns_through_windows(hq, hk, d, b, window, dtype):
    """Windows on the kernel of many columns at 128 and 256 channels too (lengths not known, so that it is taken): several tiles of
    columns a row, sight that begins past the row's first units, tokens that only some of a wave's columns see."""
    rows = [(700, 700, None), (390, 130, None), (64, 64, None), (0, 5, 0), (1000, 90, None), (333, 60, -20), (130, 70, 100)]
    check_attend(hq, hk, d, b, rows, dtype, window=window, seed=d + window)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("hq,hk,d,nq", [(8, 1, 128, 150), (4, 2, 128, 900), (6, 1, 256, 100)])
@pytest.mark.parametrize("window", [48, 500])
def test_attend_uneven_scores_through_windows(window, hq, hk, d, nq, dtype):
    """Blocks that take nearly all the weight of the queries that see them, where a window hides them from others."""
    n, b = 1500, 16
    for i, (far, size) in enumerate((([1499 - nq // 2], 1.0), ([1490], 2.0 ** -12), ([1499 - nq - window // 2, 1499 - nq // 3, 1480], 2.0 ** 12))):
        rng = np.random.default_rng(200 + i)
        q, cache, table, kv, q_off, pos = skewed_case(rng, hq, hk, d, b, n, nq, dtype, far, size)
        scale = 0.5 * d ** -0.5
        want, mag, dots, top = E.attend(host(q), cache, table, kv, q_off, pos, scale, window)
        with ctx_of(hq, hk, d, b, cache.n, table.shape[1], dtype) as ctx:
            for max_kv in (n, 0):
                got = host(pkg.kv_attend(ctx, q, dev(cache.bytes), dev(table), dev(kv), dev(q_off), dev(pos), scale=scale, window=window,
                                         max_q=nq, max_kv=max_kv))
                lim = bound(dtype, want, mag, dots, d, n, top)
                assert (np.abs(got - want) <= lim).all(), (far, max_kv, float((np.abs(got - want) / lim).max()))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("window", [20, 70])
def test_attend_through_windows_beside_garbage(window, dtype):
    """... and blocks before every window that hold no numbers."""
    test_attend_beside_garbage(4, 1, 128, 16, 150, window, dtype)
