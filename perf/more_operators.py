"""The 8-bit cache of a replica and the pages that its requests share, as timed cases.

A replica's cache of keys and values may hold 8-bit codes with a scale for each block and kv head
in place of 4-bit ones with a scale for each token:
  store    norms and rotates the queries and keys of new tokens and writes keys and values to their
           slots, in blocks that may hold earlier tokens; what those blocks hold is read back,
  attend   lets the new tokens' queries attend to the cache.
Requests of one workflow begin alike, and their rows may share the blocks of what they have in common:
  fork     rows that begin with the first tokens of other rows; partly filled blocks are copied,
  release  rows give up their blocks; those that nobody holds any more are free,
  compact  all blocks in use move to the front, so that the end of the cache can be given back.

Cell of a block (B tokens of D channels) and kv head: key codes [B][D], value codes [B/4][D][4] (four
tokens of a channel side by side), fp32 scales of keys and of values, 8 bytes unused.  A code is e4m3
(sign, 4 bits of exponent, 3 of mantissa, no infinity); a value is its code's value times the scale, a power of two
2^e, e the least for which no magnitude in the block passes 448 * 2^e (-100 at least, 119 at most).  Storing at a block's first
token starts it anew; otherwise its scale never falls, and where it rises the codes it holds are rounded to the new one.
"""
import math
import random

import torch

own = False

DEVICE = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
E4M3 = torch.float8_e4m3fn
POSITIONS = 40960

STORE = dict(op="store", q_heads=32, kv_heads=8, dim=128, dtype="bf16", block=16, tokens=1, rows=1,
             norm=True, rot=128, pairs=False, mix=1)
ATTEND = dict(op="attend", q_heads=32, kv_heads=8, dim=128, dtype="bf16", block=16, rows=1, context=1024,
              queries=1, window=0, refused=0, mix=1)
FORK = dict(op="fork", kv_heads=8, dim=128, codes="e4m3", block=16, layers=1, rows=16, forks=4, sources=1, context=1000, spare=120, mix=1)
RELEASE = dict(op="release", block=16, rows=16, context=1000, group=1, released=20, mix=1)
COMPACT = dict(op="compact", kv_heads=8, dim=128, codes="e4m3", block=16, layers=1, rows=16, context=1000, keep=70, mix=1)


def listed():
    return [
        # a decode step: a token for each request, interleaved rotation of half the channels
        dict(STORE, name="store_decode", q_heads=14, kv_heads=2, dim=64, dtype="f16", block=32, tokens=181, rows=181,
             norm=False, rot=32, pairs=True),
        # a large batch of prompt tokens, every row from the middle of a block on
        dict(STORE, name="store_prompts", q_heads=40, block=64, tokens=14000, rows=9),
        # a decode step over ragged contexts
        dict(ATTEND, name="attend_decode", rows=80, context=5000),
        # one request with a very long context: few rows, a long axis
        dict(ATTEND, name="attend_long", q_heads=40, dtype="f16", block=64, context=150001),
        # a whole prompt at once
        dict(ATTEND, name="attend_prompt", block=64, context=7001, queries=7001),
        # chunks of prompts against their contexts, a sliding window, one request refused its blocks
        dict(ATTEND, name="attend_chunks", q_heads=14, kv_heads=2, dim=64, dtype="f16", block=32, rows=7,
             context=8000, queries=500, window=4096, refused=1),
        # an agent asks four others with what it has so far
        dict(FORK, name="fork_few", layers=4, context=2001),
        # many requests begin with a few long texts, blocks short at the end
        dict(FORK, name="fork_many", block=32, layers=4, rows=700, forks=250, sources=9, context=8000, spare=90),
        # a few requests of a batch end
        dict(RELEASE, name="release_few", rows=64, context=4000, released=6),
        # the largest batch, rows in groups that share what they begin with
        dict(RELEASE, name="release_many", rows=1500, context=6000, group=6, released=35),
        # a small replica (4-bit codes) gives a third of its blocks back
        dict(COMPACT, name="compact_small", kv_heads=2, dim=64, codes="e2m1", rows=24, context=700),
        # a large one makes room for another model
        dict(COMPACT, name="compact_large", block=32, layers=2, rows=96, context=3000, keep=80),
    ]


HEADS = ((32, 8, 128), (40, 8, 128), (16, 8, 128), (14, 2, 64), (64, 8, 128), (12, 12, 64), (8, 4, 256), (71, 1, 64))
BLOCKS = (16, 32, 64, 128)


def draw(rng):
    def size(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    mix, block = rng.randrange(1 << 20), rng.choice(BLOCKS)
    shape = dict(zip(("q_heads", "kv_heads", "dim"), rng.choice(HEADS)))
    op = rng.choice(("store", "store", "attend", "attend", "attend", "fork", "release", "compact"))
    if op == "store":
        tokens = size(1, 8000)
        rot = shape["dim"] // rng.choice((1, 2, 4))
        return {**STORE, **shape, "dtype": rng.choice(("bf16", "f16")), "block": block, "mix": mix, "tokens": tokens,
                "rows": rng.choice((1, max(1, tokens // 100), tokens)), "norm": rng.random() < 0.7, "rot": rot,
                "pairs": rng.random() < 0.3}
    if op == "attend":
        base = {**ATTEND, **shape, "dtype": rng.choice(("bf16", "f16")), "block": block, "mix": mix}
        if rng.random() < 0.6:   # single tokens
            case = {**base, "context": size(1, 150001), "window": rng.choice((0, 0, 1000))}
            most = min(256, 700000000 // (case["context"] * case["kv_heads"] * case["dim"]))
            return {**case, "rows": size(1, max(1, most))}
        context = size(2, 9000)
        case = {**base, "context": context, "queries": min(context, size(2, 4000)), "window": rng.choice((0, 0, 500)),
                "refused": rng.choice((0, 1))}
        most = 1000000000 // (case["context"] * case["queries"] * case["q_heads"])
        return {**case, "rows": max(1 + case["refused"], min(most, size(1, 32)))}
    if op == "release":
        context = size(1, 20000)
        return {**RELEASE, "block": block, "mix": mix, "context": context, "rows": size(1, min(1500, max(1, 20000000 // context))),
                "group": rng.choice((1, 2, 6)), "released": rng.choice((3, 30, 100))}
    heads = {"kv_heads": shape["kv_heads"], "dim": shape["dim"], "codes": rng.choice(("e4m3", "e2m1")), "block": block, "mix": mix,
             "layers": rng.choice((1, 2, 5))}
    context = size(1, 20000)
    token = heads["layers"] * heads["kv_heads"] * heads["dim"] * 2
    most = 300000000 // (token * (context + block))          # rows that the cache has room for
    if op == "fork":
        forks = size(1, max(1, min(300, 150000000 // (token * block))))
        return {**FORK, **heads, "context": context, "forks": forks, "sources": max(1, min(most, forks // rng.choice((1, 4, 30)))),
                "rows": 2 * forks + size(1, 300), "spare": rng.choice((80, 120))}
    return {**COMPACT, **heads, "context": context, "rows": size(1, max(1, min(most, 500))), "keep": rng.choice((60, 80, 95))}


# ---- sizes that follow from a case -------------------------------------------------------------

def blocks_of(n, block):
    return -(-n // block)


def attend_rows(case):
    """(tokens in the cache, queries) of each row; the first is the largest."""
    r = random.Random(case["mix"])
    rows = [(case["context"], case["queries"])]
    while len(rows) < case["rows"]:
        kv = r.randint(max(1, case["context"] // 8), case["context"])
        rows.append((kv, min(kv, r.randint(1, case["queries"]))))
    for k in range(case["refused"]):
        rows[-1 - k] = (0, rows[-1 - k][1])
    return rows


def fork_rows(case):
    """Tokens that each row holds (the sources first, then the rows that forks fill, then others), and (source, row, tokens) of each fork."""
    r = random.Random(case["mix"])
    held = [r.randint(max(1, case["context"] // 2), case["context"]) for _ in range(case["sources"])]
    first = len(held)
    rows = max(case["rows"], first + case["forks"])
    held += [0] * case["forks"] + [r.randint(0, 3 * case["block"]) for _ in range(rows - first - case["forks"])]
    forks = []
    for k in range(case["forks"]):
        source = k * first // case["forks"]
        # most go on from all that the source holds, some from an earlier point
        forks.append((source, first + k, held[source] if r.random() < 0.7 else r.randint(1, held[source])))
    r.shuffle(forks)
    return held, forks


def fork_room(case):
    """Free blocks of a fork's case, and the forks that get the block they need (or need none)."""
    _, forks = fork_rows(case)
    needs = [int(n % case["block"] > 0) for _, _, n in forks]
    free = sum(needs) * case["spare"] // 100 + 1
    upto, got = 0, []
    for need in needs:
        upto += need
        got.append(not need or upto <= free)
    return free, got


def release_rows(case):
    """Tokens that each row holds, the blocks it shares with the others of its group, and whether it ends."""
    r, b = random.Random(case["mix"]), case["block"]
    held = [r.randint(1, case["context"]) for _ in range(case["rows"])]
    common = []
    for k in range(0, len(held), case["group"]):
        group = held[k:k + case["group"]]
        common += [r.randint(0, min(n // b for n in group)) if len(group) > 1 else 0] * len(group)
    ends = [r.random() * 100 < case["released"] for _ in held]
    ends[r.randrange(len(held))] = True
    return held, common, ends


def compact_rows(case):
    """Tokens that each row holds, the blocks in use, those of the cache and those kept."""
    r = random.Random(case["mix"])
    held = [r.randint(1, case["context"]) for _ in range(case["rows"])]
    used = sum(blocks_of(n, case["block"]) for n in held)
    keep = used + 1 + used // 20
    return held, used, max(keep + 1, keep * 100 // case["keep"]), keep


def cell_bytes(case):
    b, d = case["block"], case["dim"]
    return 2 * b * d + 16 if case.get("codes", "e4m3") == "e4m3" else b * (d + 4)


def work(case):
    b = case["block"]
    if case["op"] == "fork":
        held, forks = fork_rows(case)
        free, got = fork_room(case)
        blocks = sum(blocks_of(n, b) for n in held) + free
        copies = sum(g and n % b > 0 for g, (_, _, n) in zip(got, forks))
        entries = sum(blocks_of(n, b) for g, (_, _, n) in zip(got, forks) if g)
        return {"bytes": 2 * copies * case["layers"] * case["kv_heads"] * cell_bytes(case) + 8 * blocks + 8 * len(held) + 8 * entries +
                len(forks) * 21, "flops": 0}
    if case["op"] == "release":
        held, common, ends = release_rows(case)
        given = sum(blocks_of(n, b) for n, e in zip(held, ends) if e)
        blocks = sum(blocks_of(n, b) for n in held) - sum(c for k, c in enumerate(common) if k % case["group"])
        return {"bytes": 8 * blocks + 9 * len(held) + 8 * given, "flops": 0}
    if case["op"] == "compact":
        held, used, total, keep = compact_rows(case)
        moved = used * (total - keep) // total
        return {"bytes": 2 * moved * case["layers"] * case["kv_heads"] * cell_bytes(case) + 12 * keep + 4 * (total - used) + 8 * used +
                8 * min(keep, total - keep) + 4 * len(held), "flops": 0}
    hq, hk, d = case["q_heads"], case["kv_heads"], case["dim"]
    if case["op"] == "store":
        t = case["tokens"]
        moved = t * (2 * hq + 2 * hk) * d * 2            # q in and out, k and v in
        moved += t * 2 * hk * d * 2                      # written, and read back
        moved += t * 2 * hk * d * 2 + t * 20             # values read back, positions and slots
        moved += min(t, POSITIONS) * case["rot"] * 4
        return {"bytes": moved, "flops": t * (hq + 2 * hk) * d * 8}
    seen = pairs = tokens = 0
    for kv, q in attend_rows(case):
        tokens += q
        if kv:
            first = kv - q                               # the first query's position
            w = case["window"] or kv
            seen += kv - max(0, first - w + 1)
            a = max(0, min(q, w - first))                # queries whose window reaches the start
            pairs += a * (first + 1) + a * (a - 1) // 2 + (q - a) * w
    return {"bytes": seen * 2 * hk * d + 2 * tokens * hq * d * 2 + blocks_of(seen, b) * (4 + 8 * hk) + 12 * tokens,
            "flops": 4 * d * hq * pairs}


# ---- inputs ------------------------------------------------------------------------------------

def ints(x, dtype=torch.int32):
    return torch.tensor(x, dtype=dtype, device=DEVICE)


def tables(held, common, group, b, ids, width):
    """Block tables of rows that hold `held` tokens, the first `common` blocks of each group's rows the same ones; the ids in use and
    how many more rows hold each."""
    have = (ints(held) + b - 1) // b
    common = ints(common)
    row = torch.arange(len(held), device=DEVICE)
    lead = row // group * group
    mine = torch.where(row == lead, have, have - common)
    first = mine.cumsum(0) - mine
    at = torch.arange(width, device=DEVICE)[None]
    theirs = at < torch.where(row == lead, 0, common)[:, None]
    place = torch.where(theirs, first[lead][:, None] + at, first[:, None] + at - torch.where(row == lead, 0, common)[:, None])
    table = torch.where(at < have[:, None], ids[place.clamp(0, ids.numel() - 1)], -1).int()
    more = torch.zeros(ids.numel(), dtype=torch.int32, device=DEVICE)
    more.scatter_add_(0, torch.where(theirs, table, 0).long().flatten(), theirs.int().flatten())
    return table, int(mine.sum()), more


def ring_of(ids, used, r):
    """Ring and pool of the blocks that are not in use."""
    total, free = ids.numel(), ids.numel() - used
    head = r.randrange(total)
    ring = torch.full((total,), -1, dtype=torch.int32, device=DEVICE)
    ring[(head + torch.arange(free, device=DEVICE)) % total] = ids[used:]
    return ring, ints([head, free])


def prepare(case, seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    r = random.Random(seed)
    state = {"case": case}
    b = case["block"]
    if case["op"] in ("fork", "release", "compact"):
        common, group = None, 1
        if case["op"] == "fork":
            held, forks = fork_rows(case)
            total = sum(blocks_of(n, b) for n in held) + fork_room(case)[0]
            order = list(range(len(held)))
            r.shuffle(order)                             # rows in any order
            held, new = [held[k] for k in order], {k: i for i, k in enumerate(order)}
            state.update(src=ints([new[s] for s, _, _ in forks]), dst=ints([new[d] for _, d, _ in forks]), count=ints([n for _, _, n in forks]))
        elif case["op"] == "release":
            held, common, ends = release_rows(case)
            group = case["group"]
            total = sum(blocks_of(n, b) for n in held) + 7
            state.update(ends=ints(ends, torch.uint8))
        else:
            held, _, total, state["keep"] = compact_rows(case)
            r.shuffle(held)
        width = max(blocks_of(n, b) for n in held) + 2
        if case["op"] == "release":                      # as many blocks as are held, and a few free ones
            total -= sum(c for k, c in enumerate(common) if k % group)
        ids = torch.randperm(total, generator=g, device=DEVICE).int()
        table, used, shared = tables(held, common or [0] * len(held), group, b, ids, width)
        ring, pool = ring_of(ids, used, r)
        state.update(lens=ints(held), table=table, shared=shared, ring=ring, pool=pool)
        if case["op"] != "release":
            state["cache"] = torch.randint(0, 256, (case["layers"], total, case["kv_heads"] * cell_bytes(case)), generator=g,
                                           device=DEVICE, dtype=torch.uint8)
        return state
    hq, hk, d, dt = case["q_heads"], case["kv_heads"], case["dim"], TYPES[case["dtype"]]

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=DEVICE)

    def filled(total):
        """A cache that holds normal values, of another size in each block."""
        cache = torch.zeros(total, hk, 2 * b * d + 16, dtype=torch.uint8, device=DEVICE)
        step = max(1, (1 << 26) // (hk * b * d))
        for at in range(0, total, step):                 # in parts that fit beside the cache
            k, v, s = parts(cache[at:at + step], b, d)
            for i, to in enumerate((k, v)):
                x = normal(s.shape[0], hk, b, d) * torch.exp(0.4 * normal(s.shape[0], hk, 1, 1))
                s[..., i] = power(least_power(x.abs().amax((-1, -2))))
                x = (x / s[..., i, None, None]).to(E4M3).view(torch.uint8)
                to[:] = x.unflatten(-2, (b // 4, 4)).transpose(-1, -2) if i else x
        return cache

    if case["op"] == "store":
        t, n = case["tokens"], case["rows"]
        sizes = [t // n + (k < t % n) for k in range(n)]
        at_mix = random.Random(case["mix"])              # (so that as many earlier tokens come back for every seed)
        starts = [at_mix.randrange(1, POSITIONS - s) for s in sizes]
        row = torch.repeat_interleave(torch.arange(n, device=DEVICE), ints(sizes))
        first = ints([0] + sizes[:-1]).cumsum(0)
        pos = ints(starts)[row] + torch.arange(t, device=DEVICE) - first[row]
        begin = ints([s // b for s in starts])
        count = ints([blocks_of(s + m, b) - s // b for s, m in zip(starts, sizes)])
        total = int(count.sum()) + 3
        ids = torch.randperm(total, generator=g, device=DEVICE)
        slot = ids[(count.cumsum(0) - count)[row] + pos // b - begin[row]] * b + pos % b
        # what the first blocks held before, and the new tokens
        open_row = torch.repeat_interleave(torch.arange(n, device=DEVICE), ints([s % b for s in starts]))
        open_at = torch.cat([torch.arange(s % b) for s in starts]).to(DEVICE)
        back = torch.cat([ids[(count.cumsum(0) - count)[open_row]] * b + open_at, slot])
        spread = torch.exp(0.5 * normal((hq + 2 * hk) * d))   # activations of a layer: channels of different sizes
        qkv = (normal(t, (hq + 2 * hk) * d) * spread).to(dt)
        angle = torch.arange(POSITIONS, device=DEVICE)[:, None] * 1e6 ** (-torch.arange(0, case["rot"], 2, device=DEVICE) / case["rot"])
        state.update(qkv=qkv, pos=pos.int(), slot=slot, back=back, cos_sin=torch.cat([angle.cos(), angle.sin()], 1).float().contiguous(),
                     q_weight=(1 + 0.3 * normal(d)).to(dt), k_weight=(1 + 0.3 * normal(d)).to(dt), cache=filled(total))
        return state
    rows = attend_rows(case)
    r.shuffle(rows)
    width = max(1, max(blocks_of(kv, b) for kv, _ in rows))
    lens, count = ints([kv for kv, _ in rows]), ints([q for _, q in rows])
    q_off = torch.cat([count.new_zeros(1), count.cumsum(0)]).long()
    t = sum(q for _, q in rows)
    row = torch.repeat_interleave(torch.arange(len(rows), device=DEVICE), count)
    pos = torch.arange(t, device=DEVICE) - q_off[row] + (lens[row] - count[row]).clamp(min=0)
    ids = torch.randperm(sum(blocks_of(kv, b) for kv, _ in rows) + 2, generator=g, device=DEVICE).int()
    table, _, _ = tables([kv for kv, _ in rows], [0] * len(rows), 1, b, ids, width)
    state.update(cache=filled(ids.numel()), table=table, lens=lens, q_off=q_off.int(), pos=pos.int(), scale=d ** -0.5,
                 q=(1.5 * normal(t, hq, d)).to(dt), max_q=max(q for _, q in rows), max_kv=max(kv for kv, _ in rows))
    return state


def parts(cells, b, d):
    """Key codes [.., B, D], value codes [.., B/4, D, 4] and scales [.., 2] of cells, as views."""
    n = b * d
    return (cells[..., :n].unflatten(-1, (b, d)), cells[..., n:2 * n].unflatten(-1, (b // 4, d, 4)), cells[..., 2 * n:2 * n + 8].view(torch.float32))


def least_power(most):
    """The least e for which `most` (fp32, finite) does not pass 448 * 2^e = 1.75 * 2^(e + 8), from -100 to 119; from its bits, so exactly."""
    u = most.contiguous().view(torch.int32)
    return ((u >> 23) - 127 - 8 + ((u & 0x7fffff) > 0x600000)).clamp(-100, 119)


def power(e):
    return ((e + 127) << 23).int().view(torch.float32)


# ---- one pass ----------------------------------------------------------------------------------

_contexts = {}


def context(state):
    """The handle that a replica keeps for its cache: one for each geometry."""
    case = state["case"]
    cache, table = state.get("cache"), state.get("table")
    blocks = state["ring"].numel() if "ring" in state else cache.shape[0]
    key = (case.get("q_heads", case.get("kv_heads", 1)), case.get("kv_heads", 1), case.get("dim", 64), case["block"], case.get("dtype", "bf16"),
           case.get("codes", "e4m3"), blocks, 1 if table is None else table.shape[1])
    if key not in _contexts:
        import paper_2609_03335_amd as wf
        _contexts[key] = wf.KVContext(0, q_heads=key[0], kv_heads=key[1], head_dim=key[2], block_tokens=key[3], dtype=key[4],
                                      codes=key[5], n_blocks=key[6], max_blocks=key[7])
    return _contexts[key]


def run(state):
    case = state["case"]
    if own:
        import paper_2609_03335_amd as wf
        ctx = context(state)
        if case["op"] == "fork":
            lens, pool, shared, granted, moves = wf.kv_fork(ctx, state["src"], state["dst"], state["count"], state["lens"], state["pool"],
                                                            state["ring"], state["table"], state["shared"])
            wf.kv_copy(ctx, state["cache"], moves, layers=case["layers"])
            return {"lens": lens, "pool": pool, "shared": shared, "granted": granted, "moves": moves, "table": state["table"],
                    "cache": state["cache"]}
        if case["op"] == "release":
            lens, pool, shared = wf.kv_release(ctx, state["ends"], state["lens"], state["pool"], state["ring"], state["table"], state["shared"])
            return {"lens": lens, "pool": pool, "shared": shared, "ring": state["ring"]}
        if case["op"] == "compact":
            pool, ring, shared, done, moves = wf.kv_compact(ctx, state["keep"], state["lens"], state["pool"], state["ring"], state["table"],
                                                            state["shared"])
            wf.kv_copy(ctx, state["cache"], moves, layers=case["layers"])
            return {"pool": pool, "ring": ring, "shared": shared, "done": done, "moves": moves, "table": state["table"], "cache": state["cache"]}
        if case["op"] == "store":
            q, k, v = heads_of(state)
            q = wf.kv_store(ctx, q, k, v, state["pos"], state["slot"], state["cache"], state["cos_sin"], rot_dim=case["rot"],
                            interleaved=case["pairs"], q_weight=state["q_weight"] if case["norm"] else None,
                            k_weight=state["k_weight"] if case["norm"] else None, eps=1e-6)
            k, v = wf.kv_load(ctx, state["cache"], state["back"])
            return {"q": q, "k": k, "v": v}
        return wf.kv_attend(ctx, state["q"], state["cache"], state["table"], state["lens"], state["q_off"], state["pos"],
                            scale=state["scale"], window=case["window"], max_q=state["max_q"], max_kv=state["max_kv"])
    return {"fork": plain_fork, "release": plain_release, "compact": plain_compact, "store": plain_store, "attend": plain_attend}[case["op"]](state)


def plain_fork(state):
    b, lens, table, ring, shared, cache = (state["case"]["block"], *(state[k] for k in ("lens", "table", "ring", "shared", "cache")))
    src, dst = state["src"].long(), state["dst"].long()
    head, free, total = state["pool"][0], state["pool"][1], ring.numel()
    n = torch.minimum(state["count"], lens[src])
    full, rest = n // b, n % b > 0
    upto = rest.int().cumsum(0)
    granted = (lens[dst] == 0) & (~rest | (upto <= free))
    got = granted & rest
    fresh = torch.where(got, ring[(head + upto - 1) % total], -1)
    at = torch.arange(table.shape[1], device=table.device)[None]
    common = (at < full[:, None]) & granted[:, None]
    row = torch.where(common, table[src], torch.where((at == full[:, None]) & got[:, None], fresh[:, None], table[dst]))
    new_table = table.clone()
    new_table[dst] = row
    more = torch.cat([shared, shared.new_zeros(1)]).scatter_add(0, torch.where(common, table[src], total).long().flatten(),
                                                                 common.int().flatten())[:total]
    old = torch.where(got, table[src, full.clamp(max=table.shape[1] - 1).long()], -1)
    cache[:, fresh[got].long()] = cache[:, old[got].long()]
    new_lens = lens.clone()
    new_lens[dst] = torch.where(granted, n, lens[dst]).int()
    return {"lens": new_lens, "pool": torch.stack([(head + got.sum()) % total, free - got.sum()]).int(), "shared": more, "granted": granted.byte(),
            "moves": torch.stack([old, fresh]).int(), "table": new_table, "cache": cache}


def plain_release(state):
    b, lens, table, ring, shared = (state["case"]["block"], *(state[k] for k in ("lens", "table", "ring", "shared")))
    head, free, total = state["pool"][0], state["pool"][1], ring.numel()
    ends = state["ends"] != 0
    at = torch.arange(table.shape[1], device=table.device)[None]
    given = ends[:, None] & (at < ((lens + b - 1) // b)[:, None])
    left = torch.cat([shared, shared.new_zeros(1)]).scatter_add(0, torch.where(given, table, total).long().flatten(), -given.int().flatten())[:total]
    over = left < 0
    place = torch.where(over, (head + free + over.cumsum(0) - 1) % total, total).long()
    new_ring = torch.cat([ring, ring.new_zeros(1)]).scatter(0, place, torch.arange(total, device=ring.device).int())[:total]
    return {"lens": torch.where(ends, 0, lens), "pool": torch.stack([head, free + over.sum()]).int(), "shared": left.clamp(min=0), "ring": new_ring}


def plain_compact(state):
    b, keep, lens, table, ring, shared, cache = (state["case"]["block"], *(state[k] for k in ("keep", "lens", "table", "ring", "shared", "cache")))
    head, free, total = state["pool"][0], state["pool"][1], ring.numel()
    ids = torch.arange(total, device=ring.device)
    idle = torch.zeros(total + 1, dtype=torch.bool, device=ring.device)
    idle[torch.where(ids < free, ring[(head + ids) % total], total).long()] = True
    idle = idle[:total]
    # the k-th block in use behind the kept ones goes to the k-th free one of these
    goes, hole = ~idle & (ids >= keep), idle & (ids < keep)
    most = min(keep, total - keep)
    moved = goes.sum()
    moves = torch.full((2, most + 1), -1, dtype=torch.int32, device=ring.device)
    moves[0, torch.where(goes, goes.cumsum(0) - 1, most)] = ids.int()
    place = hole.cumsum(0) - 1
    taken = hole & (place < moved)
    moves[1, torch.where(taken, place, most)] = ids.int()
    moves = moves[:, :most]
    to = ids.clone()
    here = moves[0] >= 0
    to[moves[0][here].long()] = moves[1][here].long()
    new_ring = torch.full((keep + 1,), -1, dtype=torch.int32, device=ring.device)
    new_ring[torch.where(hole & ~taken, place - moved, keep)] = ids.int()
    new_shared = torch.where(idle, 0, shared)[:keep]
    new_shared[moves[1][here].long()] = shared[moves[0][here].long()]
    at = torch.arange(table.shape[1], device=table.device)[None]
    mine = at < ((lens + b - 1) // b)[:, None]
    new_table = torch.where(mine, to[table.clamp(min=0).long()], table).int()
    cache[:, moves[1][here].long()] = cache[:, moves[0][here].long()]
    left = (hole & ~taken).sum()
    return {"pool": torch.stack([torch.zeros_like(left), left]).int(), "ring": new_ring[:keep], "shared": new_shared,
            "done": torch.ones(1, dtype=torch.int32, device=ring.device), "moves": moves, "table": new_table, "cache": cache}


def heads_of(state):
    case = state["case"]
    hq, hk, d = case["q_heads"], case["kv_heads"], case["dim"]
    x = state["qkv"]
    return (x[:, :hq * d].unflatten(-1, (hq, d)), x[:, hq * d:(hq + hk) * d].unflatten(-1, (hk, d)), x[:, (hq + hk) * d:].unflatten(-1, (hk, d)))


def rotated(x, cos, sin, rot, pairs):
    """x [T, H, D] with its first `rot` channels rotated: halves (c, c + rot/2), or neighbours (2c, 2c+1)."""
    cos, sin, h = cos[:, None], sin[:, None], rot // 2
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if pairs else (x[..., :h], x[..., h:rot])
    y, z = a * cos - b * sin, b * cos + a * sin
    both = torch.stack([y, z], -1).flatten(-2) if pairs else torch.cat([y, z], -1)
    return torch.cat([both, x[..., rot:]], -1)


def squares(x):
    """Sum of squares over the last axis, neighbours added first: the same to the last bit on both sides, so that no code is off by one."""
    x = x * x
    while x.shape[-1] > 1:
        x = x[..., 0::2] + x[..., 1::2]
    return x


def plain_store(state):
    case, dt = state["case"], state["qkv"].dtype
    b, d, rot = case["block"], case["dim"], case["rot"]
    q, k, v = (x.float() for x in heads_of(state))
    if case["norm"]:
        q = q * torch.rsqrt(squares(q) * (1.0 / d) + 1e-6) * state["q_weight"].float()
        k = k * torch.rsqrt(squares(k) * (1.0 / d) + 1e-6) * state["k_weight"].float()
    cos, sin = state["cos_sin"][state["pos"]].split(rot // 2, -1)
    q, k = rotated(q, cos, sin, rot, case["pairs"]), rotated(k, cos, sin, rot, case["pairs"])
    keys, values, scales = parts(state["cache"], b, d)
    block, off = state["slot"] // b, state["slot"] % b
    n, hk = scales.shape[:2]
    # blocks that get tokens, and those that hold earlier ones
    begin = torch.full((n,), b, dtype=torch.int64, device=off.device).scatter_reduce(0, block, off, "amin")
    at = block[:, None].expand(-1, hk)
    for i, (x, codes) in enumerate(((k, keys), (v, values))):
        most = x.new_zeros(n, hk).scatter_reduce(0, at, x.abs().amax(-1), "amax")
        old = scales[..., i]
        e = (old.contiguous().view(torch.int32) >> 23) - 127
        need = least_power(most)
        new = power(torch.where((begin == b)[:, None], e, torch.where((begin == 0)[:, None], need, torch.maximum(e, need))))
        keep = (begin > 0)[:, None] & (begin < b)[:, None] & (new != old)
        held = (codes.view(E4M3).float() * (old / new)[..., None, None] if i == 0 else codes.view(E4M3).float() * (old / new)[..., None, None, None])
        codes[:] = torch.where(keep.view(n, hk, *[1] * (codes.dim() - 2)), held.to(E4M3).view(torch.uint8), codes)
        scales[..., i] = new
        code = (x / new[block][..., None]).clamp(-448, 448).to(E4M3).view(torch.uint8)
        if i == 0:
            codes[block, :, off] = code
        else:
            codes[block, :, off // 4, :, off % 4] = code
    # read back
    block, off = state["back"] // b, state["back"] % b
    most = torch.finfo(dt).max
    k = keys[block, :, off].view(E4M3).float() * scales[block, :, 0, None]
    v = values[block, :, off // 4, :, off % 4].view(E4M3).float() * scales[block, :, 1, None]
    return {"q": q.to(dt), "k": k.clamp(-most, most).to(dt), "v": v.clamp(-most, most).to(dt)}


def plain_attend(state):
    case, q = state["case"], state["q"]
    b, d, hk, g = case["block"], case["dim"], case["kv_heads"], case["q_heads"] // case["kv_heads"]
    rows, nq, nk = len(state["lens"]), state["max_q"], max(1, state["max_kv"])
    cells = state["cache"][state["table"][:, :blocks_of(nk, b)].clamp(min=0)]        # [R, blocks, Hk, cell]
    keys, values, scales = parts(cells, b, d)
    keys = (keys.view(E4M3).float() * scales[..., 0, None, None]).permute(0, 2, 4, 1, 3).reshape(rows, hk, d, -1)
    values = (values.view(E4M3).float() * scales[..., 1, None, None, None]).permute(0, 2, 1, 3, 5, 4).reshape(rows, hk, -1, d)
    # the packed queries, padded to rows
    off = state["q_off"].long()
    i = torch.arange(nq, device=q.device)[None]
    at = (off[:-1, None] + i).clamp(max=len(q) - 1)
    pos = torch.where(i < (off[1:] - off[:-1])[:, None], state["pos"][at], -1)
    x = q[at].float().view(rows, nq, hk, g, d).permute(0, 2, 3, 1, 4).reshape(rows, hk, g * nq, d)
    s = torch.matmul(x, keys).view(rows, hk, g, nq, -1) * state["scale"]
    j = torch.arange(s.shape[-1], device=q.device)
    see = (j <= pos[..., None]) & (j < state["lens"][:, None, None])
    if case["window"]:
        see &= j > pos[..., None] - case["window"]
    s = torch.where(see[:, None, None], s, -torch.inf)
    m = s.amax(-1, keepdim=True)
    s = torch.exp(s - torch.where(m == -torch.inf, 0, m))
    total = s.sum(-1, keepdim=True)
    s = s / torch.where(total == 0, 1, total)
    o = torch.matmul(s.view(rows, hk, g * nq, -1), values).view(rows, hk, g, nq, d).permute(0, 3, 1, 2, 4).reshape(rows * nq, hk * g, d)
    token = torch.arange(len(q), device=q.device)
    row = torch.searchsorted(off[1:], token, right=True)
    return o[row * nq + token - off[row]].to(q.dtype)


# ---- the definition in 64 bits -----------------------------------------------------------------

def two_to(e):
    """Exactly (powers of a library may be off by a last bit, which moves values that are half-way between two codes)."""
    return (e.long() + 1023 << 52).view(torch.float64)


def code_value(c):
    """Values of e4m3 codes from their bits."""
    c = c.int()
    e, m = c >> 3 & 15, (c & 7).double()
    return torch.where(e > 0, (1 + m / 8) * two_to(e - 7), m / 512) * (1 - 2 * (c >> 7).double())


def on_grid(y, s):
    """y rounded to the values that codes of scale s stand for: gaps of an eighth of a power of two, of 2^-9 at the low end."""
    u = y.abs() / s
    gap = two_to(torch.frexp(u.clamp(min=2.0 ** -6))[1] - 4)
    return (u / gap).round().mul(gap).clamp(max=448) * y.sign() * s


def exact(case, seed):
    if case["op"] not in ("store", "attend"):
        return None                                      # whole numbers
    state = prepare(case, seed)
    b, d, hq, hk = case["block"], case["dim"], case["q_heads"], case["kv_heads"]
    if case["op"] == "store":
        x = state["qkv"].double().view(case["tokens"], hq + 2 * hk, d)
        angle_c, angle_s = state["cos_sin"].double()[state["pos"]].chunk(2, -1)
        z = torch.complex(angle_c, angle_s)[:, None]
        out = {}
        blocks, where = torch.unique(state["slot"] // b, return_inverse=True)
        back = state["back"]
        n_old = back.numel() - case["tokens"]
        for name, part in (("q", x[:, :hq]), ("k", x[:, hq:hq + hk]), ("v", x[:, hq + hk:])):
            y = part
            if name != "v":
                if case["norm"]:
                    y = y / (y.pow(2).mean(-1, keepdim=True) + 1e-6).sqrt() * state[name + "_weight"].double()
                r, h = case["rot"], case["rot"] // 2
                turn = y[..., :r].unflatten(-1, (h, 2)) if case["pairs"] else y[..., :r].unflatten(-1, (2, h)).transpose(-1, -2)
                turn = torch.view_as_real(torch.complex(turn[..., 0], turn[..., 1]) * z)
                turn = turn.flatten(-2) if case["pairs"] else turn.transpose(-1, -2).flatten(-2)
                y = torch.cat([turn, y[..., r:]], -1)
            if name != "q":
                i = int(name == "v")
                scale = state["cache"][..., 2 * b * d:].contiguous().view(torch.float32)[..., i].double()      # [blocks, Hk]
                most = torch.zeros(blocks.numel(), hk, dtype=torch.float64, device=DEVICE)
                most.index_reduce_(0, where, y.abs().amax(-1), "amax")
                starts = torch.zeros(blocks.numel(), device=DEVICE).index_add_(0, where, (state["slot"] % b == 0).float()) > 0
                m, x2 = torch.frexp(most)                # 448 * 2^e is 0.875 * 2^(e + 9)
                new = two_to((x2 - 9 + (m > 0.875)).clamp(-100, 119))
                new = torch.where(starts[:, None], new, torch.maximum(new, scale[blocks]))
                fresh = on_grid(y, new[where][..., None])
                if n_old:
                    at, off = back[:n_old] // b, (back[:n_old] % b)[:, None]
                    c = torch.arange(d, device=DEVICE)[None]
                    byte = off * d + c if i == 0 else b * d + (off // 4 * d + c) * 4 + off % 4
                    held = code_value(state["cache"][at].gather(2, byte[:, None].expand(-1, hk, -1))) * scale[at][..., None]
                    held = on_grid(held, new[torch.searchsorted(blocks, at)][..., None])
                    fresh = torch.cat([held, fresh])
                y = fresh
            out[name] = y
        return out
    heads = state["q"].double().view(-1, hk, hq // hk, d)
    out = torch.zeros(heads.shape, dtype=torch.float64, device=DEVICE)
    off, lens = state["q_off"].tolist(), state["lens"].tolist()
    for n, kv in enumerate(lens):
        if not kv or off[n] == off[n + 1]:
            continue
        cells = state["cache"][state["table"][n, :blocks_of(kv, b)]].transpose(0, 1)    # [Hk, blocks, cell]
        scale = cells[..., 2 * b * d:].contiguous().view(torch.float32).double()
        pos = state["pos"][off[n]:off[n + 1]].long()[:, None]
        j = torch.arange(kv, device=DEVICE)[None]
        hide = (j > pos) | ((j <= pos - case["window"]) if case["window"] else j < 0)
        for h in range(hk):
            k = (code_value(cells[h, :, :b * d]) * scale[h, :, :1]).reshape(-1, d)[:kv]
            v = code_value(cells[h, :, b * d:2 * b * d]) * scale[h, :, 1:2]
            v = v.reshape(-1, d, 4).transpose(1, 2).reshape(-1, d)[:kv]
            for i in range(hq // hk):
                s = (heads[off[n]:off[n + 1], h, i] @ k.T * state["scale"]).masked_fill(hide, -math.inf)
                out[off[n]:off[n + 1], h, i] = torch.softmax(s, -1).nan_to_num(0) @ v
    return out.view(-1, hq, d)
