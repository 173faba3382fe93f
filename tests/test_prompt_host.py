"""CPU checks of the entry points of include/moeflow_prompt.h: the declared symbols
are exported, invalid arguments are rejected on the host before a device is touched,
workspace sizes never fall, and the oracle's pins."""
import ctypes
import itertools
import os
import re

import numpy as np
import pytest
import torch

import oracle
from paper_2410_17954_amd import ops
from paper_2410_17954_amd.build import library_path

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "moeflow_prompt.h")
BIG = 1 << 40
NAN, INF = float("nan"), float("inf")


def at(i):
    """Addresses far from each other, never dereferenced: validation fails first."""
    return ctypes.c_void_p((i + 1) << 44)


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(library_path()):
        from paper_2410_17954_amd import build
        build.build(verbose=False)
    return ops.load_library()


def test_every_declared_symbol_is_exported(lib):
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = re.findall(r"^\s*(?:const\s+)?\w+\*?\s+\*?(moe_\w+)\s*\(", text, re.M)
    assert sorted(names) == sorted(ops.exported_prompt_symbols())
    for n in names:
        assert hasattr(lib, n)


def _prompt(lib, q=at(0), k=at(1), v=at(2), dt=1, N=4096, M=4096, B=1, Hq=8, Hkv=2, D=64, qs=None,
            ks=None, vs=None, qo=at(3), ko=at(4), scale=0.125, out=at(5), lse=at(6), ws=at(7),
            nbytes=-1):
    # nbytes -1: too small where any workspace is needed
    qs = Hq * D if qs is None else qs
    ks = Hkv * D if ks is None else ks
    vs = Hkv * D if vs is None else vs
    return lib.moe_prompt_attention(q, k, v, dt, N, M, B, Hq, Hkv, D, qs, ks, vs, qo, ko, scale, out,
                                    lse, ws, BIG if nbytes < 0 else nbytes, None)


def test_prompt_attention_rejects_bad_arguments(lib):
    S = None
    for bad in (dict(q=S), dict(k=S), dict(v=S), dict(out=S), dict(dt=2), dict(N=0), dict(M=-1),
                dict(B=0), dict(Hq=0), dict(Hkv=0), dict(Hq=9), dict(D=0), dict(qs=511),
                dict(ks=127), dict(vs=120), dict(qo=S, B=2), dict(ko=S, B=2, M=4095),
                dict(scale=NAN), dict(scale=INF), dict(scale=2.4e38),
                dict(out=at(0)), dict(out=at(1)), dict(out=at(3)), dict(lse=at(5)), dict(lse=at(2)),
                dict(out=ctypes.c_void_p((1 << 44) + 4096)),
                dict(q=ctypes.c_void_p(at(5).value - 16))):
        assert _prompt(lib, **bad) == ops.MOE_ERR_ARG, bad
    odd = ctypes.c_void_p((9 << 44) + 8)
    for bad in (dict(D=60), dict(D=264), dict(q=odd), dict(k=odd), dict(v=odd), dict(out=odd),
                dict(qs=516), dict(ks=132, vs=132), dict(dt=0, qs=514), dict(vs=(1 << 24) + 8),
                dict(M=1 << 31), dict(N=1 << 28), dict(B=1 << 31), dict(B=1 << 22, Hkv=1, Hq=4)):
        assert _prompt(lib, **bad) == ops.MOE_ERR_UNSUPPORTED, bad


def _store(lib, load=False, k=at(0), v=at(1), dt=1, N=16, Hkv=2, D=64, ks=128, vs=128, slots=at(2),
           n_slots=20, kc=at(3), ksc=at(4), vc=at(5), vsc=at(6)):
    if load:
        return lib.moe_kv4_load(kc, ksc, vc, vsc, n_slots, slots, N, Hkv, D, dt, ks, vs, k, v, None)
    return lib.moe_kv4_store(k, v, dt, N, Hkv, D, ks, vs, slots, n_slots, kc, ksc, vc, vsc, None)


@pytest.mark.parametrize("load", [False, True])
def test_kv4_store_and_load_reject_bad_arguments(lib, load):
    S = None
    for bad in (dict(k=S), dict(v=S), dict(kc=S), dict(ksc=S), dict(vc=S), dict(vsc=S), dict(dt=2),
                dict(N=0), dict(n_slots=0), dict(Hkv=0), dict(D=0), dict(ks=127), dict(vs=120),
                dict(slots=S, N=21), dict(k=at(3)), dict(v=at(6)),
                dict(kc=ctypes.c_void_p(at(0).value + 16 * 256 - 16))):
        assert _store(lib, load, **bad) == ops.MOE_ERR_ARG, bad
    if load:
        assert _store(lib, load, v=at(0)) == ops.MOE_ERR_ARG
        inside = ctypes.c_void_p(at(0).value + 272)      # ends in the next token's keys
        assert _store(lib, load, v=inside, ks=256, vs=256) == ops.MOE_ERR_ARG
    else:
        assert _store(lib, load, vc=at(3)) == ops.MOE_ERR_ARG
        assert _store(lib, load, ksc=at(2)) == ops.MOE_ERR_ARG
    odd = ctypes.c_void_p((9 << 44) + 8)
    for bad in (dict(D=48), dict(D=288, ks=576, vs=576), dict(k=odd), dict(v=odd), dict(kc=odd),
                dict(vc=odd), dict(ks=132), dict(dt=0, vs=130), dict(vs=(1 << 24) + 8),
                dict(N=1 << 30), dict(n_slots=1 << 31),
                dict(N=1 << 27, n_slots=1 << 27)):
        assert _store(lib, load, **bad) == ops.MOE_ERR_UNSUPPORTED, bad


def _attend(lib, q=at(0), dt=1, R=4, Hq=8, Hkv=2, D=64, kc=at(1), ks=at(2), vc=at(3), vs=at(4), C=4,
            S=1000, row=at(5), lens=at(6), scale=0.125, out=at(7), lse=at(8), ws=at(9), nbytes=BIG):
    return lib.moe_kv4_attention(q, dt, R, Hq, Hkv, D, kc, ks, vc, vs, C, S, row, lens, scale, out,
                                 lse, ws, nbytes, None)


def test_kv4_attention_rejects_bad_arguments(lib):
    S = None
    for bad in (dict(q=S), dict(out=S), dict(kc=S), dict(ks=S), dict(vc=S), dict(vs=S), dict(dt=2),
                dict(R=0), dict(C=0), dict(S=0), dict(Hq=0), dict(Hkv=0), dict(Hq=9), dict(D=0),
                dict(row=S, R=5), dict(scale=NAN), dict(scale=-INF), dict(scale=2.4e38),
                dict(out=at(0)), dict(lse=at(7)), dict(out=at(1)), dict(lse=at(6))):
        assert _attend(lib, **bad) == ops.MOE_ERR_ARG, bad
    odd = ctypes.c_void_p((12 << 44) + 8)
    for bad in (dict(D=48), dict(D=288), dict(q=odd), dict(out=odd), dict(kc=odd), dict(vc=odd),
                dict(S=1 << 31), dict(C=1 << 31), dict(R=1 << 29), dict(R=1 << 21),
                dict(Hq=1 << 19, Hkv=1 << 19, R=1)):
        assert _attend(lib, **bad) == ops.MOE_ERR_UNSUPPORTED, bad


def _logprobs(lib, z=at(0), dt=1, R=3, V=1000, stride=1000, tok=at(1), m=2, n=4, lp=at(2), en=at(3),
              tt=at(4), tl=at(5), ws=at(6), nbytes=BIG):
    return lib.moe_token_logprobs(z, dt, R, V, stride, tok, m, n, lp, en, tt, tl, ws, nbytes, None)


def test_token_logprobs_rejects_bad_arguments(lib):
    S = None
    odd = ctypes.c_void_p((9 << 44) + 1)
    for bad in (dict(z=S), dict(tok=S), dict(lp=S), dict(tt=S), dict(tl=S), dict(dt=2), dict(R=0),
                dict(V=0), dict(m=-1), dict(n=-1), dict(stride=999), dict(z=odd),
                dict(m=0, n=0, en=S), dict(lp=at(0)), dict(en=at(2)), dict(tt=at(1)),
                dict(tl=at(4))):
        assert _logprobs(lib, **bad) == ops.MOE_ERR_ARG, bad
    for bad in (dict(n=65), dict(V=(1 << 24) + 1, stride=1 << 25), dict(R=1 << 22),
                dict(m=1 << 30), dict(stride=1 << 31)):
        assert _logprobs(lib, **bad) == ops.MOE_ERR_UNSUPPORTED, bad


def test_workspaces_are_needed_and_refused(lib):
    need = lib.moe_prompt_attention_workspace(64, 30000, 1, 8, 2, 64, 1)
    few = dict(N=64, M=30000)
    if need:
        for bad in (dict(ws=None), dict(nbytes=need - 1), dict(ws=ctypes.c_void_p((8 << 44) + 16))):
            assert _prompt(lib, **few, **bad) == ops.MOE_ERR_WORKSPACE, bad
    need = lib.moe_kv4_attention_workspace(4, 1000, 8, 2, 64)
    if need:
        for bad in (dict(ws=None), dict(nbytes=need - 1), dict(ws=ctypes.c_void_p((10 << 44) + 16))):
            assert _attend(lib, **bad) == ops.MOE_ERR_WORKSPACE, bad
        assert _attend(lib, out=at(9)) == ops.MOE_ERR_ARG
    need = lib.moe_token_logprobs_workspace(3, 100000, 2, 4)
    if need:
        for bad in (dict(ws=None), dict(nbytes=need - 1), dict(ws=ctypes.c_void_p((7 << 44) + 16))):
            assert _logprobs(lib, V=100000, stride=100000, **bad) == ops.MOE_ERR_WORKSPACE, bad
    assert lib.moe_prompt_attention_workspace(0, 5, 1, 8, 2, 64, 1) == 0
    assert lib.moe_kv4_attention_workspace(4, 1000, 8, 3, 64) == 0
    assert lib.moe_token_logprobs_workspace(3, 100, 2, 65) == 0


def _never_falls(size, *axes):
    grid = {p: size(*(a[i] for a, i in zip(axes, p)))
            for p in itertools.product(*(range(len(a)) for a in axes))}
    for p, n in grid.items():
        for d in range(len(p)):
            q = p[:d] + (p[d] + 1,) + p[d + 1:]
            if q in grid:
                assert n <= grid[q], [(a[i], a[j]) for a, i, j in zip(axes, p, q)]


@pytest.mark.parametrize("Hq,Hkv,D", [(32, 8, 128), (16, 16, 64), (8, 1, 256), (64, 2, 96), (3, 3, 32)])
def test_workspace_of_the_largest_call_serves_all(lib, Hq, Hkv, D):
    N = list(range(1, 40)) + [63, 64, 65, 127, 128, 129, 500, 1000, 4096, 16384]
    M = [0, 1, 64, 127, 128, 500, 4096, 30000, 300000]
    for dt in (0, 1):
        for B in (1, 3, 64):
            _never_falls(lambda n, m: ops.prompt_attention_workspace(n, m, B, Hq, Hkv, D, dt), N, M)
        _never_falls(lambda n, b: ops.prompt_attention_workspace(n, 5000, b, Hq, Hkv, D, dt), N[::5],
                     list(range(1, 70)))
    _never_falls(lambda r, s: ops.kv4_attention_workspace(r, s, Hq, Hkv, D), list(range(1, 140)) + [500, 4000],
                 [1, 31, 32, 33, 127, 128, 129, 500, 4096, 65536, 1 << 20])


def test_logprobs_workspace_of_the_largest_call_serves_all(lib):
    _never_falls(lambda r, v, n: ops.token_logprobs_workspace(r, v, 1, n),
                 list(range(1, 70)) + [127, 128, 129, 255, 256, 257, 1000, 5000],
                 [1, 500, 2047, 2048, 2049, 4096, 16384, 16385, 32000, 50257, 128000, 152000, 1 << 20],
                 [0, 1, 4, 16, 20, 64])


# ------------------------------------------------------------------ oracle pins
def test_oracle_prompt_closed_forms():
    g = np.random.default_rng(1)
    q, k, v = (g.normal(size=(5, h, 8)) for h in (4, 2, 2))
    out, lse = oracle.prompt_attention(q, k, v, [0, 3, 5], [0, 3, 5], 0.3)
    # a first token sees itself only
    for t in (0, 3):
        assert np.allclose(out[t, 2], v[t, 1]) and np.allclose(lse[t, 2], 0.3 * q[t, 2] @ k[t, 1])
    # the last token of a sequence is decode attention over all of its keys
    a, b = oracle.prefix_attention(q[2:3], k[None, :3], v[None, :3], [3], k[None, :0], v[None, :0], [0],
                                   [0, 1], 0.3)
    assert np.allclose(out[2], a[0]) and np.allclose(lse[2], b[0])
    # a chunk gives what the whole gave
    c, d = oracle.prompt_attention(q[1:3], k[:3], v[:3], [0, 2], [0, 3], 0.3)
    assert np.allclose(c, out[1:3]) and np.allclose(d, lse[1:3])
    # more queries than keys: the first have none; a row of no sequence is kept
    c, d = oracle.prompt_attention(q, k[:2], v[:2], [0, 4], [0, 2], 0.0, np.ones(q.shape), np.ones((5, 4)))
    assert not c[:2].any() and (d[:2] == -np.inf).all() and (c[4] == 1).all() and (d[4] == 1).all()
    assert np.allclose(c[3, :2], v[:2, 0].mean(0)) and np.allclose(d[3], np.log(2))


def test_oracle_kv4_encoding():
    x = np.zeros((3, 64))
    x[0, :8] = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0]       # ties: the even code
    x[0, 8:11] = [-0.26, -0.0, 6.9]
    x[0, 32] = 7.5                                                # past 7: the next power
    x[1, 0], x[1, 33] = 2.0 ** -140, 3.4e38
    x[2, 5], x[2, 40] = np.nan, -np.inf
    codes, scales = oracle.kv4_encode(x)
    assert scales.tolist() == [[127, 128], [3, 252], [255, 255]]
    flat = np.stack([codes & 15, codes >> 4], -1).reshape(3, 64)
    assert flat[0, :11].tolist() == [0, 2, 2, 4, 4, 6, 6, 7, 9, 8, 7]
    assert flat[0, 32] == 6 and flat[1, 0] == 0 and flat[1, 33] == 7 and not flat[2].any()
    y = oracle.kv4_decode(codes, scales)
    assert y[0, :8].tolist() == [0, 1, 1, 2, 2, 4, 4, 6] and y[0, 32] == 8
    assert y[1, 33] == 6 * 2.0 ** 125 and np.isnan(y[2]).all()
    # every value a block holds is held again by itself
    again = oracle.kv4_decode(*oracle.kv4_encode(y[:2]))
    assert np.array_equal(again, y[:2])


def test_oracle_kv4_attention_is_attention_over_the_values():
    g = np.random.default_rng(2)
    k, v = g.normal(size=(2, 2, 6, 2, 32))
    cache = oracle.kv4_encode(k) + oracle.kv4_encode(v)
    q = g.normal(size=(3, 4, 32))
    out, lse = oracle.kv4_attention(q, cache, [1, 5, 0], [4, 6, 0], 0.2)
    kk, vv = oracle.kv4_decode(*cache[:2]), oracle.kv4_decode(*cache[2:])
    a, b = oracle.prefix_attention(q[:1], kk[1:], vv[1:], [4], kk[:1, :0], vv[:1, :0], [0], [0, 1], 0.2)
    assert np.allclose(out[0], a[0]) and np.allclose(lse[0], b[0])
    assert not out[1:].any() and (lse[1:] == -np.inf).all()


def test_oracle_logprobs_closed_forms():
    z = np.array([[2.0, 1.0, 0.0, 0.0], [-np.inf, 3.0, -np.inf, 3.0]])
    p = np.exp(z) / np.exp(z).sum(1, keepdims=True)
    lp, en, top, tl = oracle.token_logprobs(z, np.array([[0, 3, 4], [1, 0, -1]]), 3)
    assert np.allclose(lp[0, :2], np.log(p[0, [0, 3]])) and lp[0, 2] == -np.inf
    assert np.allclose(lp[1, 0], np.log(0.5)) and (lp[1, 1:] == -np.inf).all()
    assert np.allclose(en, [-(p[0] * np.log(p[0])).sum(), np.log(2)])
    assert top.tolist() == [[0, 1, 2], [1, 3, -1]] and tl[1, 2] == -np.inf
    z = np.array([[-np.inf] * 3, [0.0, np.nan, 1.0], [0.0, np.inf, 1.0]])
    lp, en, top, tl = oracle.token_logprobs(z, np.zeros((3, 1), int), 2)
    assert lp[0, 0] == -np.inf and en[0] == 0 and np.isnan(lp[1:]).all() and np.isnan(en[1:]).all()
    assert (top == -1).all() and (tl == -np.inf).all()


def test_prompt_kernels_spill_nothing():
    # launches of a few microseconds, or loops whose reloads would wait on their loads
    from test_kernel_resources import _kernels
    kernels = _kernels()
    for name in ("pr_kernel", "ka_kernel", "kv4_store_kernel", "kv4_load_kernel", "lp_kernel",
                 "attention_join_kernel"):
        mine = {n: (k[".vgpr_spill_count"], k[".private_segment_fixed_size"])
                for n, k in kernels.items() if name in n}
        assert mine, name
        assert not {n: v for n, v in mine.items() if any(v)}


def test_tensors_of_the_host_are_refused(lib):
    """In the first place too: what a check of one device compares the others with."""
    x, q = torch.zeros((2, 4, 64)), torch.zeros((2, 4, 64))
    i = lambda *v: torch.tensor(v, dtype=torch.int32)
    cache = tuple(torch.zeros((1, 8, 4, w), dtype=torch.uint8) for w in (32, 2, 32, 2))
    k4 = torch.zeros((2, 3, 4, 64))
    w = torch.zeros((4, 8, 16))
    for call in (lambda: ops.prompt_attention(q, x, x), lambda: ops.kv4_store(x, x, cache),
                 lambda: ops.kv4_load(cache), lambda: ops.kv4_load(cache, k=x, v=x),
                 lambda: ops.kv4_attention(x[:1], cache),
                 lambda: ops.token_logprobs(x[0], i(1, 2, 3, 4).view(4, 1)),
                 lambda: ops.prefix_attention(q, k4, k4),
                 lambda: ops.layer_decode(torch.zeros((2, 16)), torch.zeros((4, 16)), w, w,
                                          w.transpose(1, 2).contiguous(), 2),
                 lambda: ops.beam_select(torch.zeros((1, 2, 9)), torch.zeros((1, 2))),
                 lambda: ops.beam_reorder([torch.zeros((1, 2, 3, 8))], i(0, 1).view(1, 2))):
        with pytest.raises(ValueError, match="on the GPU"):
            call()
