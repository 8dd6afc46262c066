"""The serving example: planned activations served over the paged 4-bit cache,
each step's attention against a 64-bit one over what the cache holds."""
import importlib.util
import os

import numpy as np
import pytest
import torch

import paper_2609_03335_amd as pkg

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "serve_activations.py")


@pytest.fixture(scope="module")
def example():
    assert torch.cuda.is_available(), "GPU tests need a HIP device"
    spec = importlib.util.spec_from_file_location("serve_activations", PATH)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def requests(example, replica, most_prompt=90, most_answer=8):
    rng = np.random.default_rng(3)
    activations = example.granted_activations()
    assert activations
    return [(rng.integers(0, 997, int(rng.integers(1, most_prompt))).tolist(), int(rng.integers(1, most_answer)))
            for _ in activations[:20]]


@pytest.mark.parametrize("window", [0, 30])
def test_every_step_attends_to_what_is_stored(example, monkeypatch, window):
    """All requests end, every block comes back, and each layer's attention is that over
    the tokens stored so far (in 64 bits, from kv_load)."""
    replica = example.Replica(rows=5, layers=2, q_heads=8, kv_heads=2, head_dim=64, blocks=30, row_blocks=8, window=window)
    ctx, real, seen = replica.ctx, pkg.kv_attend, []

    def checked(c, q, cache, table, lens, q_off, pos, **kw):
        out = real(c, q, cache, table, lens, q_off, pos, **kw)
        n, off = lens.tolist(), q_off.tolist()
        for r in range(len(n)):
            if off[r] == off[r + 1] or n[r] == 0:
                continue
            j = torch.arange(n[r], device=q.device)
            k, v = (x.double().repeat_interleave(4, 1) for x in pkg.kv_load(c, cache, table[r].long()[j // 16] * 16 + j % 16))
            p = pos[off[r]:off[r + 1]].long()
            see = j[None] <= p[:, None]
            if window:
                see &= j[None] > p[:, None] - window
            s = (q[off[r]:off[r + 1]].double().transpose(0, 1) @ k.permute(1, 2, 0).contiguous()) * kw["scale"]
            w = torch.softmax(s.masked_fill(~see[None], -torch.inf), -1).nan_to_num(0)
            want, size = (w @ y.transpose(0, 1).contiguous() for y in (v, v.abs()))
            got = out[off[r]:off[r + 1]].double().transpose(0, 1)
            # loads are rounded to bf16 (2^-8 of a key's products with the query, which move p by as much), p and
            # the output once more
            move = (q[off[r]:off[r + 1]].double().abs().transpose(0, 1) @ k.abs().permute(1, 2, 0).contiguous()).amax(-1, keepdim=True)
            lim = (4 * 2.0 ** -8 + 2.2 * 2.0 ** -9 * kw["scale"] * move) * size + 1e-6
            assert bool(((got - want).abs() <= lim).all())
            seen.append(off[r + 1] - off[r])
        return out

    monkeypatch.setattr(example.wf, "kv_attend", checked)
    jobs = requests(example, replica)
    answers = example.serve(replica, jobs, chunk=40)
    assert [len(a) for a in answers] == [count for _, count in jobs]
    assert all(0 <= t < 997 for a in answers for t in a)
    assert max(seen) > 16 and min(seen) == 1
    # a last step releases nothing: all blocks are in the ring, each once
    assert replica.pool[1].item() == 30 and sorted(replica.ring.tolist()) == list(range(30))
    assert replica.lens.tolist() == [0] * 5
    replica.close()


def test_answers_do_not_depend_on_the_blocks(example):
    """Requests one after the other in one call and in a call each, on caches whose blocks come
    in another order."""
    replica = lambda: example.Replica(rows=1, layers=2, q_heads=8, kv_heads=2, head_dim=64, blocks=30, row_blocks=8)
    a, b = replica(), replica()
    b.ring = b.ring.flip(0).contiguous()
    jobs = requests(example, a)[:4]
    one = example.serve(a, jobs, chunk=32)
    again = [example.serve(b, [job], chunk=32)[0] for job in jobs]
    assert one == again
    a.close()
    b.close()


def test_too_small_a_cache_is_an_error(example):
    replica = example.Replica(rows=2, layers=1, q_heads=4, kv_heads=2, head_dim=64, blocks=2, row_blocks=8)
    with pytest.raises(RuntimeError):
        example.serve(replica, [([1] * 60, 2)])
    replica.close()
