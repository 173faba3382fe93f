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
