"""Host-side checks of the 8-bit cache and of shared pages (no GPU): geometry, refusals, the oracle's own
codes and page operators."""
import ctypes
import os

import numpy as np
import pytest

import kv8_oracle as E
import paper_2609_03335_amd as pkg
from paper_2609_03335_amd import _lib

GOOD = dict(q_heads=8, kv_heads=2, head_dim=64, block_tokens=16, n_blocks=10, max_blocks=4, dtype="bf16")


@pytest.fixture(scope="module", autouse=True)
def built():
    if not os.path.exists(_lib.LIB_PATH):
        from paper_2609_03335_amd import build
        build.build()


def test_cache_bytes():
    # a token of a head: D bytes of key codes, as many of values; 16 bytes for the scales of a block
    assert pkg.wf_kv_cache_bytes(**GOOD, codes="e4m3") == 10 * 2 * (16 * 64 * 2 + 16)
    assert pkg.wf_kv_cache_bytes(**dict(GOOD, dtype=pkg.WF_KV_F16 | pkg.WF_KV_E4M3)) == 10 * 2 * (16 * 64 * 2 + 16)
    assert pkg.wf_kv_cache_bytes(**GOOD, codes="e2m1") == pkg.wf_kv_cache_bytes(**GOOD)
    big = dict(GOOD, n_blocks=1 << 22, kv_heads=8, head_dim=128, block_tokens=64, codes="e4m3")
    assert pkg.wf_kv_cache_bytes(**big) == (1 << 22) * 8 * (64 * 256 + 16)   # past 32 bits


@pytest.mark.parametrize("bad", [dict(dtype=2 | 16), dict(dtype=32), dict(dtype=-1), dict(head_dim=96), dict(block_tokens=8)])
def test_bad_geometry_is_refused(bad):
    with pytest.raises(pkg.WFError):
        pkg.wf_kv_cache_bytes(**{**GOOD, **bad}, codes="e4m3")


def test_unknown_codes_are_refused():
    with pytest.raises(ValueError):
        pkg.wf_kv_cache_bytes(**GOOD, codes="e5m2")


def test_null_contexts():
    lib = _lib.load()
    assert lib.wf_kv_fork(None, None, None, None, 0, 0, *[None] * 13) == pkg.WF_EINVAL
    assert lib.wf_kv_release(None, None, 0, *[None] * 10) == pkg.WF_EINVAL
    assert lib.wf_kv_compact(None, 1, 0, *[None] * 14) == pkg.WF_EINVAL
    assert lib.wf_kv_copy(None, None, 0, 1, None, None, 0, None) == pkg.WF_EINVAL
    assert b"NULL" in lib.wf_kv_last_error(None)


def test_oracle_codes_are_the_nearest():
    assert E.VALUES[0x7e] == 448 and E.VALUES[1] == 2.0 ** -9 and np.isnan(E.VALUES[0x7f]) and E.VALUES[0x38] == 1
    rng = np.random.default_rng(0)
    x = np.concatenate([rng.standard_normal(3000) * 2.0 ** rng.integers(-12, 9, 3000), [0, 448, 464, 1e9, 2.0 ** -10, 3 * 2.0 ** -10]])
    x = np.concatenate([x, -x])
    every = E.VALUES[np.isfinite(E.VALUES)]
    got = E.VALUES[E.codes(x)]
    assert np.array_equal(np.abs(got - np.clip(x, -448, 448)), np.abs(every[None] - np.clip(x, -448, 448)[:, None]).min(-1))
    # ties to the even code: 17 is between 16 and 18, 19 between 18 and 20; half the least value goes to 0
    assert list(E.VALUES[E.codes(np.array([17.0, 19, 21, 2.0 ** -10, 3 * 2.0 ** -10, 5 * 2.0 ** -10]))]) == [16, 20, 20, 0, 2.0 ** -8, 2.0 ** -8]


def test_oracle_least_power():
    for e in range(-100, 120):
        top = 448 * 2.0 ** e
        assert E.least_power(top) == e and E.least_power(np.nextafter(top, 0)) == e
        assert E.least_power(np.nextafter(top, np.inf)) == min(e + 1, 119)
    assert E.least_power(0) == -100 and E.least_power(3e38) == 119


def test_oracle_blocks_grow():
    """A block's scale follows its largest magnitude, never falls while it grows, and begins anew at its first token."""
    rng = np.random.default_rng(1)
    c = E.Cache8(2, 1, 16, 64)
    x = rng.standard_normal((16, 2, 1, 64)).astype(np.float32)
    c.put([16], x[0, :1], x[0, 1:])
    small = c.scales()[1, 0, 0]
    c.put([17, 18], 40 * x[1:3, 0], x[1:3, 1])
    assert c.scales()[1, 0, 0] > small
    k, v = c.get([16, 17, 18])
    for got, want, s in ((k[0], x[0, 0], c.scales()[1, 0, 0]), (k[1], 40 * x[1, 0], c.scales()[1, 0, 0]), (v[2], x[2, 1], c.scales()[1, 0, 1])):
        # half a step: 2^-4 of the value, or half the least code; the first token was rounded twice
        assert (np.abs(got - want) <= 2.2 * (2.0 ** -4 * np.abs(want) + 2.0 ** -10 * s)).all()
    c.put([16], x[0, :1], x[0, 1:])
    assert c.scales()[1, 0, 0] == small


def test_oracle_pages_keep_their_counts():
    """Forks, releases and a compaction in turn: every block is free once, or held by as many rows as are counted."""
    rng = np.random.default_rng(2)
    b, n, rows, width = 16, 60, 12, 8
    lens, pool, ring = np.zeros(rows, int), np.array([0, n]), np.arange(n)
    table, shared = np.full((rows, width), -1), np.zeros(n, int)

    def check():
        held = np.zeros(len(ring), int)
        for r in range(rows):
            for j in range(-(-int(lens[r]) // b)):
                held[table[r, j]] += 1
        free = [int(ring[(pool[0] + i) % len(ring)]) for i in range(pool[1])]
        assert len(set(free)) == len(free) and all(held[x] == 0 for x in free)
        assert np.array_equal(np.maximum(held - 1, 0), shared) and (held > 0).sum() + len(free) == len(ring)

    for i in range(200):
        if i == 120:
            used = n - pool[1]
            keep = max(int(used), 40)
            s = E.compact(keep, lens, pool, ring, table, shared, b)
            assert s["done"][0] == 1
            pool, ring, shared, table = s["pool"], s["ring"], s["shared"], s["table"]
        elif rng.random() < 0.4:
            f = [(int(rng.integers(0, rows)), d, int(rng.integers(0, 130))) for d in rng.permutation(rows)[:3]]
            s = E.fork(f, lens, pool, ring, table, shared, b)
            lens, pool, shared, table = s["lens"], s["pool"], s["shared"], s["table"]
        elif rng.random() < 0.5:
            ends = rng.random(rows) < 0.2
            s = E.release(ends, lens, pool, ring, table, shared, b)
            lens, pool, shared, ring = s["lens"], s["pool"], s["shared"], s["ring"]
        else:
            import kv_oracle as K
            s = K.step(rng.integers(0, 40, rows), lens, pool, ring, table, b, 0)
            lens, pool, ring, table = s["lens"], s["pool"], s["ring"], s["table"]
        check()


def context_without_a_gpu(n_blocks):
    """A context whose calls of the library are recorded, over host tensors."""
    import torch

    class Library:
        made = []

        def wf_kv_copy(self, handle, cache, step, layers, *rest):
            self.made.append((step, layers))
            return pkg.WF_OK

        def wf_kv_ctx_destroy(self, handle):
            pass

    ctx = pkg.KVContext.__new__(pkg.KVContext)
    ctx.lib, ctx.handle, ctx.device, ctx._bind, ctx._current = Library(), 1, -1, None, None
    ctx.cache_bytes = pkg.wf_kv_cache_bytes(**dict(GOOD, n_blocks=n_blocks), codes="e4m3")
    return ctx, torch.full((2, 3), -1, dtype=torch.int32)


def test_copies_go_to_the_layers_of_a_larger_cache():
    """A context of fewer blocks goes on with the front of each layer's cache: the layers of that tensor are as far apart as they were."""
    import torch
    whole = pkg.wf_kv_cache_bytes(**GOOD, codes="e4m3")
    ctx, moves = context_without_a_gpu(4)
    part = ctx.cache_bytes
    zeros = lambda *shape: torch.zeros(shape, dtype=torch.uint8)
    for cache, layers, apart in ((zeros(3, whole), 3, whole), (zeros(2, whole), 2, whole), (zeros(3, 10, whole // 10), 3, whole),
                                 (zeros(3 * whole), 3, part), (zeros(3, part), 3, part), (zeros(5, part), 3, part),
                                 (zeros(2, 3, part), 5, part), (zeros(3 * 4, part // 4), 3, part), (zeros(3, whole), 1, part)):
        pkg.kv_copy(ctx, cache, moves, layers=layers)
        assert ctx.lib.made.pop() == (apart, layers), (tuple(cache.shape), layers)
    pkg.kv_copy(ctx, zeros(4, whole), moves, layers=2, layer_stride=whole)
    assert ctx.lib.made.pop() == (whole, 2)
    pkg.kv_copy(ctx, zeros(2, part), moves, layers=2, layer_stride=part)
    assert ctx.lib.made.pop() == (part, 2)


def test_layers_that_no_axis_shows_are_refused():
    import torch
    whole = pkg.wf_kv_cache_bytes(**GOOD, codes="e4m3")
    ctx, moves = context_without_a_gpu(4)
    zeros = lambda *shape: torch.zeros(shape, dtype=torch.uint8)
    # layers of a larger cache, more or fewer of them than are to be copied in; blocks without an axis of layers
    for cache, layers in ((zeros(4, whole), 2), (zeros(2, whole), 4), (zeros(3 * 10, whole // 10), 3), (zeros(1, 3 * whole), 3)):
        with pytest.raises(ValueError):
            pkg.kv_copy(ctx, cache, moves, layers=layers)
    with pytest.raises(ValueError):
        pkg.kv_copy(ctx, zeros(3, whole), moves, layers=3, layer_stride=2 * whole)     # past the end
    assert not ctx.lib.made


def test_blocks_of_no_context_are_refused():
    lib = _lib.load()
    assert lib.wf_kv_ctx_set_blocks(None, 4) == pkg.WF_EINVAL and b"NULL" in lib.wf_kv_last_error(None)


def test_a_context_checks_by_the_blocks_it_was_given():
    """Number of blocks and bytes of a cache follow; a refused number changes neither."""
    ctx, _ = context_without_a_gpu(10)
    asked = []
    ctx.lib.wf_kv_ctx_set_blocks = lambda handle, n: asked.append(n) or (pkg.WF_OK if 1 <= n <= 1 << 30 else pkg.WF_EINVAL)
    ctx.lib.wf_kv_last_error = lambda handle: b"refused"
    ctx.q_heads, ctx.kv_heads, ctx.head_dim, ctx.block_tokens, ctx.max_blocks = 8, 2, 64, 16, 4
    ctx.codes, ctx.dtype = "e4m3", pkg.WF_KV_BF16
    for n in (4, 10, 1, 1 << 22):
        ctx.wf_kv_ctx_set_blocks(n)
        assert ctx.n_blocks == n == asked[-1] and ctx.cache_bytes == pkg.wf_kv_cache_bytes(**dict(GOOD, n_blocks=n), codes="e4m3")
    for n in (0, -1, (1 << 30) + 1, (1 << 32) + 3, -(1 << 40)):
        with pytest.raises(pkg.WFError):
            ctx.wf_kv_ctx_set_blocks(n)
        assert ctx.n_blocks == 1 << 22 and not 1 <= asked[-1] <= 1 << 30
