"""Host-side checks of the paged-cache part of the library (no GPU): exports
and signatures follow include/wf_kv.h, geometry checks, argument errors, and
the oracle's own quantiser."""
import ctypes
import os
import re

import numpy as np
import pytest

import kv_oracle as K
import paper_2609_03335_amd as pkg
from paper_2609_03335_amd import _lib

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
TEXT = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "wf_kv.h")).read(), flags=re.S)
GOOD = dict(q_heads=8, kv_heads=2, head_dim=64, block_tokens=16, n_blocks=10, max_blocks=4, dtype="bf16")


@pytest.fixture(scope="module", autouse=True)
def built():
    if not os.path.exists(_lib.LIB_PATH):
        from paper_2609_03335_amd import build
        build.build()


def test_exports_follow_the_header():
    names = set(re.findall(r"\b(wf_kv_\w+)\s*\(", TEXT))
    assert names == set(_lib.KV_EXPORTS)
    lib = _lib.load()
    for name in names:
        params = [x for x in re.search(r"\b" + name + r"\s*\(([^)]*)\)\s*;", TEXT).group(1).split(",") if x.strip()]
        argtypes = getattr(lib, name).argtypes
        assert len(argtypes) == len(params), name
        for ctype, decl in zip(argtypes, params):
            if "*" in decl:
                assert ctype is ctypes.c_void_p or hasattr(ctype, "contents"), (name, decl)
            elif "int64_t" in decl:
                assert ctype is ctypes.c_int64, (name, decl)


@pytest.mark.parametrize("name", ["wf_kv_desc", "wf_kv_norm_rope"])
def test_structs_follow_the_header(name):
    body = re.search(r"typedef struct\s*\{([^}]*)\}\s*" + name + r"\s*;", TEXT).group(1)
    want = [re.sub(r"[\s\*]", "", d.split()[-1]) for d in body.split(";") if d.strip()]
    assert [f[0] for f in getattr(_lib, name)._fields_] == want


def test_cache_bytes():
    # a token of a head: D/2 bytes of key codes, as many of values, two scales
    assert pkg.wf_kv_cache_bytes(**GOOD) == 10 * 2 * 16 * (64 + 4)
    big = dict(GOOD, n_blocks=1 << 22, kv_heads=8, head_dim=128, block_tokens=64)
    assert pkg.wf_kv_cache_bytes(**big) == (1 << 22) * 8 * 64 * 132   # past 32 bits


@pytest.mark.parametrize("bad,status", [
    (dict(q_heads=7), 1), (dict(q_heads=0), 1), (dict(kv_heads=0), 1), (dict(q_heads=2048, kv_heads=2), 1),
    (dict(head_dim=96), 5), (dict(head_dim=0), 5), (dict(block_tokens=8), 5), (dict(block_tokens=48), 5),
    (dict(block_tokens=512), 5), (dict(n_blocks=0), 1), (dict(n_blocks=(1 << 30) + 1), 1), (dict(max_blocks=0), 1),
    (dict(max_blocks=(1 << 22) + 1), 1), (dict(block_tokens=256, max_blocks=1 << 23), 1), (dict(dtype=2), 1)])
def test_bad_geometry_is_refused(bad, status):
    with pytest.raises(pkg.WFError) as e:
        pkg.wf_kv_cache_bytes(**dict(GOOD, **bad))
    assert e.value.status == status and e.value.message


def test_null_context_and_outputs():
    lib = _lib.load()
    assert lib.wf_kv_ctx_create(0, None, None) == pkg.WF_EINVAL
    out = ctypes.c_void_p()
    assert lib.wf_kv_ctx_create(0, None, ctypes.byref(out)) == pkg.WF_EINVAL and not out
    assert lib.wf_kv_step(None, None, 0, 0, *[None] * 11) == pkg.WF_EINVAL
    assert lib.wf_kv_store(None, None, None, None, 0, 0, 0, 0, *[None] * 6) == pkg.WF_EINVAL
    assert lib.wf_kv_load(None, None, None, 0, None, None, None) == pkg.WF_EINVAL
    assert lib.wf_kv_attend(None, None, 0, 0, None, None, None, None, None, 0, 1.0, 0, 0, 0, None, None) == pkg.WF_EINVAL
    assert b"NULL" in lib.wf_kv_last_error(None)
    lib.wf_kv_ctx_destroy(None)


def test_no_gpu_context_fails_cleanly():
    import torch
    if torch.cuda.is_available():
        pytest.skip("a GPU is present")
    with pytest.raises(pkg.WFError) as e:
        pkg.KVContext(0, **GOOD)
    assert e.value.status == pkg.WF_EHIP


def test_oracle_codes_are_the_nearest():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((200, 64)).astype(np.float32)
    x[0] = 0
    x[1, 3] = np.inf
    x[2, 5] = np.nan
    code, bits = K.quantised(x)
    s = (bits.astype(np.uint32) << 16).view(np.float32).astype(np.float64)
    assert np.isnan(s[1]) and np.isnan(s[2]) and s[0] == 0
    v = K.values(code[3:]) * s[3:, None]
    every = np.concatenate([K.GRID, -K.GRID])
    best = np.abs(every[None, None] * s[3:, None, None] - x[3:, :, None]).min(-1)
    assert np.array_equal(np.abs(v - x[3:]), best)
    # ties go to the even code: 2.5 -> 2, 3.5 -> 4, 5 -> 4, 0.25 -> 0, 0.75 -> 1
    tie = np.zeros((1, 64), np.float32)
    tie[0, :7] = [6, 2.5, 3.5, 5, 0.25, 0.75, -1.75]
    assert list(K.values(K.quantised(tie)[0])[0, :7]) == [6, 2, 4, 4, 0, 1, -2]


def test_oracle_cache_round_trip():
    rng = np.random.default_rng(2)
    c = K.Cache(3, 2, 16, 64)
    k, v = rng.standard_normal((2, 2, 64)).astype(np.float32)
    c.put(37, k, v)
    gk, gv = c.get([37])
    for got, x in ((gk[0], k), (gv[0], v)):
        code, bits = K.quantised(x)
        assert np.array_equal(got, K.values(code) * (bits.astype(np.uint32) << 16).view(np.float32)[..., None])


def test_native_binding_leaves_what_it_does_not_take():
    """_kvbind takes sound GPU tensors only: None for all else, before any call."""
    import torch
    from paper_2609_03335_amd import build
    if not os.path.exists(build.BIND_PATH):
        build.build()
    from paper_2609_03335_amd import _kvbind as kb
    g = kb.geometry(0, 0, 8, 2, 64, 10, 4, 10 * 2 * 16 * 68, False)
    cache, slot, i = torch.zeros(10 * 2 * 16 * 68, dtype=torch.uint8), torch.zeros(3, dtype=torch.int64), torch.zeros(4, dtype=torch.int32)
    q = torch.zeros(3, 8, 64, dtype=torch.bfloat16)
    assert kb.load(g, 0, cache, slot) is None              # tensors of the host
    assert kb.load(g, 0, 4096, 4096) is None               # addresses
    assert kb.load(g, 0, cache) is None and kb.load() is None and kb.load(None, 0, cache, slot) is None
    assert kb.load("geometry", 0, cache, slot) is None and kb.load(g, -1, cache, slot) is None
    assert kb.step(g, 0, i, 3, i, i, i, i) is None and kb.step(g, 0, None, 1 << 40, i, i, i, i) is None
    assert kb.attend(g, 0, q, cache, i, i, i, i, 1.0, 0, 0, 0) is None
    assert kb.store(g, 0, q, q, q, i, slot, cache, None, 0, False, None, None, 1e-6) is None
    with pytest.raises(TypeError):
        kb.geometry(0)


@pytest.fixture(scope="module")
def sight(tmp_path_factory):
    """csrc/kv_sight.h, the kernels' own arithmetic, compiled for the host."""
    import subprocess
    at = tmp_path_factory.mktemp("sight")
    (at / "sight.cpp").write_text('#include "kv_sight.h"\nextern "C" void sight(int p, int len, int window, int* to) '
                                  '{ const wfkv::Sight s = wfkv::sight_of(p, len, window); to[0] = s.lo, to[1] = s.hi; }\n')
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-I", os.path.join(ROOT, "paper_2609_03335_amd", "csrc"),
                           str(at / "sight.cpp"), "-o", str(at / "sight.so")])
    lib = ctypes.CDLL(str(at / "sight.so"))

    def call(p, length, window):
        to = (ctypes.c_int * 2)()
        lib.sight(p, length, window, to)
        return to[0], to[1]
    return call


def test_sight_of_any_position_stays_in_the_row(sight):
    """Positions of a device array may be anything: no token index that follows from one (units of
    64 tokens, up to 16 units asked ahead) leaves 32 bits, and what is seen is the definition's."""
    top = 2 ** 31 - 1
    lengths = [0, 1, 63, 64, 65, 1000, 2 ** 30 - 1, 2 ** 30]
    for length in lengths:
        near = [length + x for x in (-2, -1, 0, 1, 2, 63, 64, 65)]
        for window in (0, 1, 2, 64, 1000, 2 ** 30, top - 1, top):
            for p in {-2 ** 31, -1, 0, 1, 50, *near, *(x + window for x in near), top - 512, top - 450, top - 300, top - 1, top}:
                if not -2 ** 31 <= p <= top:
                    continue
                lo, hi = sight(p, length, window)
                first, last = (max(0, p - window + 1) if window else 0), min(p, length - 1)
                assert (lo < hi) == (first <= last), (p, length, window)
                if lo < hi:
                    assert (lo, hi - 1) == (first, last), (p, length, window)
                assert 0 <= lo and 0 <= hi <= length, (p, length, window)
                assert (max(lo >> 6, (hi + 63) >> 6) + 16) << 6 < 2 ** 31, (p, length, window)


@pytest.mark.parametrize("case", ["whole", "no torch", "binding does not compile", "no host compiler"])
def test_the_library_is_built_without_the_binding(monkeypatch, tmp_path, capfd, case):
    """The C library needs hipcc alone: where torch or a host compiler for _kvbind is missing, it is built all the same,
    and a binding of an earlier build does not stay.  (Compilers that only make their output file.)"""
    import sys
    from paper_2609_03335_amd import build
    tool = tmp_path / "compiler"
    tool.write_text('#!/bin/sh\nwhile [ "$1" != -o ]; do shift; done\necho built > "$2"\n')
    tool.chmod(0o755)
    lib, bind = tmp_path / "lib.so", tmp_path / "_kvbind.so"
    monkeypatch.setattr(build, "PKG", str(tmp_path))
    monkeypatch.setattr(build, "LIB_PATH", str(lib))
    monkeypatch.setattr(build, "BIND_PATH", str(bind))
    monkeypatch.setenv("HIPCC", str(tool))
    monkeypatch.setenv("CXX", {"binding does not compile": "false", "no host compiler": str(tmp_path / "none")}.get(case, str(tool)))
    if case == "no torch":
        monkeypatch.setitem(sys.modules, "torch", None)
    bind.write_text("of an earlier build")
    assert build.build() == str(lib)
    assert lib.read_text() == "built\n"
    if case == "whole":
        assert bind.read_text() == "built\n"
    else:
        assert not bind.exists() and "_kvbind" in capfd.readouterr().err


def test_serving_refuses_an_empty_prompt():
    """The serving example: a request without a first token has nothing to be answered from."""
    import importlib.util
    spec = importlib.util.spec_from_file_location("serve_activations", os.path.join(ROOT, "examples", "serve_activations.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)

    class Replica:
        """Answers every row with the number of its step; grants all."""
        rows, steps = 2, 0

        def step(self, new, tokens, most=0):
            import torch
            self.steps += 1
            return torch.full((len(new),), self.steps), torch.tensor([int(n >= 0) for n in new])

    assert example.serve(Replica(), [([5, 6], 2), ([7], 1), ([8], 0)]) == [[1, 2], [1], []]
    replica = Replica()
    for requests in ([([], 1)], [([5], 1), ([], 2)]):
        with pytest.raises(ValueError):
            example.serve(replica, requests)
    assert replica.steps == 0
