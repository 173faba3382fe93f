"""The operators of moeflow_prompt.h where numbers end: infinite queries and values,
values near the largest numbers, log-probabilities next to 0."""
import numpy as np
import pytest
import torch

import oracle
from paper_2410_17954_amd import ops
from gpu_helpers import to_dev, to_host, vals
from prompt_helpers import check_row, draw, values

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
INF, NAN = float("inf"), float("nan")


def _dtype(dtype):
    return torch.bfloat16 if dtype == "bf16" else torch.float32


def _kv4(k, v, C=1):
    """A cache that holds k, v [C * S, Hkv, D], and the values that it stands for."""
    n, Hkv, D = k.shape
    cache = ops.kv4_cache(C, n // C, Hkv, D, DEV)
    ops.kv4_store(k, v, cache)
    held = ops.kv4_load(cache, dtype=torch.float32)
    return cache, tuple(vals(x) for x in held)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D,S", [(32, 65), (64, 50), (64, 700), (128, 300), (256, 130)])
def test_infinite_queries_over_a_cache_of_4_bits(D, S, dtype):
    g = np.random.default_rng(S)
    k, v = (to_dev(draw(g, "f32", S, 1, D)) for _ in range(2))
    k[:, 0, D - 1] = 2.0                             # held as a positive number in every key
    cache, (kk, vv) = _kv4(k, v)
    assert (kk[:, 0, D - 1] > 0).all()
    q = to_dev(draw(g, dtype, 1, 4, D))
    q[0, 0, D - 1], q[0, 1, D - 1] = -INF, INF
    q[0, 2, 3] = NAN
    if dtype == "f32":                               # a NaN whose upper half is infinity's
        q.view(torch.int32)[0, 2, 3] = 0x7f800001
    out, lse = ops.kv4_attention(q, cache, scale=0.1)
    assert (out[0, 0] == 0).all() and lse[0, 0] == -INF
    # infinity less infinity, and a NaN: no numbers
    assert torch.isnan(out[0, 1:3]).all() and torch.isnan(lse[0, 1:3]).all()
    x = vals(q)[0, 3]
    ref, rl = oracle.prompt.softmax_rows(0.1 * (kk[:, 0] @ x), vv[:, 0])
    check_row(vals(out)[0, 3], to_host(lse)[0, 3], ref, rl, x, kk[:, 0], vv[:, 0], 0.1, dtype)
    cache[3][:, ::5] = 255                           # whatever the values hold
    out, lse = ops.kv4_attention(q, cache, scale=0.1)
    assert (out[0, 0] == 0).all() and lse[0, 0] == -INF and torch.isnan(out[0, 3]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hkv,R", [(1, 512), (4, 512), (2, 3)])
def test_largest_values_of_a_cache_of_4_bits(Hkv, R, dtype):
    """One key of values up to 6 * 2^125 whose score is above those of the tiles before
    it, by less than a reference is raised for: results are finite."""
    g = np.random.default_rng(R)
    S, D, at = 1000, 64, 700
    k, v = (to_dev(draw(g, "f32", S, Hkv, D, std=s)) for s in (0.1, 1.0))
    k[:, :, 0], k[at, :, 0] = 0.0, 6.0
    v[at] = 0.0
    v[at, :, ::3], v[at, :, 33] = 6 * 2.0 ** 125, -2.0 ** 124
    cache, (kk, vv) = _kv4(k, v)
    assert np.abs(vv).max() == 6 * 2.0 ** 125 and (vv[at] == 0).any()
    q = draw(g, dtype, R, 2 * Hkv, D, std=0.1)
    t = to_dev(q)
    t[:, :, 0] = 0.85                                # 5 above the others: 2^7.3
    rows = torch.zeros(R, dtype=torch.int32, device=DEV)
    out, lse = ops.kv4_attention(t, cache, cache_row=rows, scale=1.0)
    assert torch.isfinite(out).all() and torch.isfinite(lse).all()
    for r in (0, R - 1):
        for h in range(2 * Hkv):
            x = vals(t)[r, h]
            ref, rl = oracle.prompt.softmax_rows(kk[:, h // 2] @ x, vv[:, h // 2])
            check_row(vals(out)[r, h], to_host(lse)[r, h], ref, rl, x, kk[:, h // 2], vv[:, h // 2],
                      1.0, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,D,n,m", [(4, 64, 700, 700), (2, 128, 5, 900), (64, 64, 600, 600)])
def test_largest_values_of_a_prompt(Hq, D, n, m, dtype):
    g = np.random.default_rng(n + D)
    q, k = (to_dev(draw(g, dtype, r, h, D, std=0.1)) for r, h in ((n, Hq), (m, Hq // 2)))
    v = to_dev(draw(g, dtype, m, Hq // 2, D))
    at = m // 2 + 3
    q[:, :, 0], k[:, :, 0], k[at, :, 0] = 1.0, 0.0, 5.0
    v[at, :, ::3] = 2.5e38                           # the sum over all keys stays a float32
    out, lse = ops.prompt_attention(q, k, v, scale=1.0)
    assert torch.isfinite(out).all() and torch.isfinite(lse).all()
    first = max(0, at - (m - n))
    for r in {0, max(0, first - 1), first, n // 2, n - 1}:
        for h in (0, Hq - 1):
            keys = slice(0, m - n + r + 1)
            kk, vv, x = vals(k)[keys, h // 2], vals(v)[keys, h // 2], vals(q)[r, h]
            ref, rl = oracle.prompt.softmax_rows(kk @ x, vv)
            check_row(vals(out)[r, h], to_host(lse)[r, h], ref, rl, x, kk, vv, 1.0, dtype)
