"""Plan a window, then serve the activations that the best plan gives to one
device, with continuous batching over the paged cache, in 4 or 8 bits:

    python examples/serve_activations.py [--rows 16] [--layers 4] [--blocks 160] [--codes e2m1|e4m3]

The scheduler scores the window's plans on the GPU and picks the best; the
activations of its device 0 become requests, in the order of their predicted
starts.  Every step is one kv_step for the batch and, per layer, one kv_store and
one kv_attend.  The model is a stand-in: random weights, the heads and the
rotation of a real one, no feed-forward part.
"""
import argparse
import os
import sys
import time

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2609_03335_amd as wf  # noqa: E402
from paper_2609_03335_amd import workload  # noqa: E402


class Replica:
    """A batch of `rows` requests on one GPU: their lengths, blocks and caches."""

    def __init__(self, *, rows=16, layers=4, q_heads=16, kv_heads=8, head_dim=128, block=16, blocks=160, row_blocks=64,
                 vocabulary=997, rot_dim=None, window=0, dtype="bf16", codes="e2m1", device=0, seed=0):
        self.ctx = wf.KVContext(device, q_heads=q_heads, kv_heads=kv_heads, head_dim=head_dim, block_tokens=block,
                                n_blocks=blocks, max_blocks=row_blocks, dtype=dtype, codes=codes)
        at, width, i32 = f"cuda:{device}", q_heads * head_dim, torch.int32
        self.rows, self.window, self.rot = rows, window, head_dim if rot_dim is None else rot_dim
        self.lens = torch.zeros(rows, dtype=i32, device=at)
        self.pool = torch.tensor([0, blocks], dtype=i32, device=at)
        self.ring = torch.arange(blocks, dtype=i32, device=at)
        self.table = torch.full((rows, row_blocks), -1, dtype=i32, device=at)
        self.caches = [torch.empty(self.ctx.cache_bytes, dtype=torch.uint8, device=at) for _ in range(layers)]
        g = torch.Generator(device=at)
        g.manual_seed(seed)
        t = self.ctx.torch_dtype
        weight = lambda *s: (torch.randn(*s, generator=g, device=at) * s[-1] ** -0.5).to(t)
        self.split = (q_heads * head_dim, kv_heads * head_dim, kv_heads * head_dim)
        self.qkv, self.out = ([weight(n, width) for _ in range(layers)] for n in (sum(self.split), width))
        self.norms = [torch.ones(head_dim, dtype=t, device=at) for _ in range(2)]
        self.embed = weight(vocabulary, width) * width ** 0.5
        angle = torch.arange(row_blocks * block, device=at)[:, None] * 1e4 ** (
            -torch.arange(0, self.rot, 2, device=at) / max(self.rot, 1))
        self.cos_sin = torch.cat([angle.cos(), angle.sin()], 1).contiguous()
        self.scale = head_dim ** -0.5

    def step(self, new, tokens, most=0):
        """One step: new[r] tokens of row r (below 0: the row ends), packed in
        `tokens`; `most`: the longest row after the step, if known.  Returns the next
        token of each row and which rows were granted blocks (the others' tokens come again)."""
        at = self.lens.device
        counts = torch.tensor(new, dtype=torch.int32, device=at)
        n, d = len(tokens), self.ctx.head_dim
        self.lens, self.pool, q_off, slot, pos, granted = wf.kv_step(self.ctx, counts, n, self.lens, self.pool, self.ring,
                                                                     self.table)
        if n == 0:
            return None, granted
        x = self.embed[torch.tensor(tokens, device=at)]
        for cache, qkv, out in zip(self.caches, self.qkv, self.out):
            q, k, v = (part.unflatten(-1, (-1, d)) for part in (x @ qkv.T).split(self.split, -1))
            q = wf.kv_store(self.ctx, q, k, v, pos, slot, cache, self.cos_sin, rot_dim=self.rot, q_weight=self.norms[0],
                            k_weight=self.norms[1])
            x = x + wf.kv_attend(self.ctx, q, cache, self.table, self.lens, q_off, pos, scale=self.scale, window=self.window,
                                 max_q=max(new), max_kv=most).flatten(1) @ out.T
        last = x[(q_off[1:].long() - 1).clamp(min=0)]
        return (last @ self.embed.T).argmax(-1), granted

    def close(self):
        self.ctx.close()


def serve(replica, requests, chunk=64):
    """Run (prompt, tokens to answer) requests to their end, `chunk` prompt tokens a
    step at most; returns the answers."""
    if not all(len(prompt) for prompt, _ in requests):
        raise ValueError("a prompt is empty")
    waiting, batch = list(enumerate(requests)), [None] * replica.rows
    answers = [[] for _ in requests]
    while waiting or any(batch):
        new, tokens = [], []
        for r, job in enumerate(batch):
            if job is None and waiting:
                index, (prompt, count) = waiting.pop(0)
                batch[r] = job = dict(index=index, todo=list(prompt), cached=0, left=count)
            if job is None:
                new.append(0)
            elif job["left"] == 0:
                new.append(-1)
            else:
                part = job["todo"][:chunk]
                new.append(len(part))
                tokens += part
        most = max((job["cached"] + max(n, 0) for n, job in zip(new, batch) if job), default=0)
        after, granted = replica.step(new, tokens, most)
        after, granted = [0] * len(new) if after is None else after.tolist(), granted.tolist()
        for r, ok in enumerate(granted):
            job = batch[r]
            if job is None:
                continue
            if new[r] < 0:
                batch[r] = None
            elif ok:
                job["cached"] += new[r]
                job["todo"] = job["todo"][new[r]:]
                if not job["todo"]:
                    answers[job["index"]].append(after[r])
                    job["left"] -= 1
                    job["todo"] = [after[r]]
        if not any(n < 0 or n > 0 and ok for n, ok in zip(new, granted)):
            raise RuntimeError("no request can go on: the cache needs more blocks")
    return answers


def granted_activations(device=0, config=0, plans=256):
    """Activations that the best plan of a window places on a device, by start."""
    win, batch = workload.make_config(config, n_plans=plans)
    with wf.Context(0) as ctx:
        ctx.wf_plan_upload_window(win)
        dev, prio, flags = wf.device_plans(batch, "cuda:0")
        scores, sched = wf.score_batch(ctx, dev, prio, flags, batch.n_plans, schedule=True, n_act=win.n_act, n_dev=win.n_dev)
        best = int(wf.argmin(ctx, scores, batch.n_plans).item())
    if best < 0:
        raise RuntimeError("no plan of the window is feasible")
    start = sched[0][best].cpu().numpy()[:win.n_act]
    mine = np.nonzero(batch.dev[best] == device)[0]
    return [int(i) for i in mine[np.argsort(start[mine], kind="stable")]]


def requests_of(activations, vocabulary, rng):
    """Stand-in texts: a prompt and a number of tokens to answer for each activation."""
    return [(rng.integers(0, vocabulary, int(rng.integers(1, 300))).tolist(), int(rng.integers(1, 40))) for _ in activations]


def main():
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    p.add_argument("--rows", type=int, default=16)
    p.add_argument("--layers", type=int, default=4)
    p.add_argument("--blocks", type=int, default=160)
    p.add_argument("--codes", choices=("e2m1", "e4m3"), default="e2m1")
    a = p.parse_args()
    activations = granted_activations()
    replica = Replica(rows=a.rows, layers=a.layers, blocks=a.blocks, codes=a.codes)
    requests = requests_of(activations, replica.embed.shape[0], np.random.default_rng(0))
    t0 = time.perf_counter()
    answers = serve(replica, requests)
    t = time.perf_counter() - t0
    print(f"{len(activations)} activations, {sum(len(x) for x, _ in requests)} prompt tokens, "
          f"{sum(map(len, answers))} answered in {t:.2f} s; free blocks {replica.pool[1].item()} of {a.blocks}")
    replica.close()


if __name__ == "__main__":
    main()
