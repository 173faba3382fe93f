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
    x = vals(q[0, 3])
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


def _check_logprobs(x, tokens, n_top, dtype):
    """Rows of numbers and -inf (float64 of the exact logits). With d = max - z, u =
    2^-24, the exponential of a logit is off by
    * 2.25 max(d, 8) u: its difference to a reference at most 8 below it or d above it is
      rounded, the factor log2 e, and their product;
    * 2 u of the exponential itself, 3 u at each change of reference (d / 8 in a thread,
      of the thread, the wave and the block), 32 u of a float32 sum of 32 terms,
    relative to p = e^-d / sum. Where the sum is below 2 terms of the maximum (d = 0) are
    exact, a sum apart: |d ln sum| <= sum of p times those over the others, and what is too
    small for a float32. The entropy's second sum has them times |z - ref| + |ref - max| <=
    max(d, 8) + d + 8 and 2 u d more. Every result is rounded once; the reference, float64
    sums and a logarithm of numbers next to 1, is off by some 2^-51."""
    u = 2.0 ** -24
    z = torch.from_numpy(x).to(_dtype(dtype)).to(DEV)
    x = vals(z)
    rl, re, rt, rtl = oracle.token_logprobs(x, tokens, n_top)
    d = x.max(1, keepdims=True) - x
    p = np.exp(-d)
    p /= p.sum(1, keepdims=True)
    fin = np.where(np.isfinite(d), d, 0.0)
    exact = np.exp(-d).sum(1, keepdims=True) < 1.99
    rest = np.where((d > 0) & np.isfinite(d) | ~exact & (d == 0), p, 0.0)
    rel = u * (2.25 * np.maximum(fin, 8) + 2 + 3 * (fin / 8 + 3) + 32) * 1.01
    e_ln = (rest * rel).sum(1) + x.shape[1] * 2.0 ** -126 + 2.0 ** -50
    e_h = (rest * (rel * (np.maximum(fin, 8) + fin + 8) + 2 * u * fin)).sum(1)
    lp, en, tt, tl = (to_host(a).astype(np.float64) for a in ops.token_logprobs(
        z, to_dev(tokens.astype(np.int32)), n_top))
    for got, ref, bound in ((lp, rl, e_ln[:, None]), (tl, rtl, e_ln[:, None]),
                            (en, re, e_ln * (1 + (rest * fin).sum(1)) + e_h)):
        ok = np.broadcast_to(np.isfinite(ref), ref.shape)
        assert np.array_equal(np.isfinite(got), ok)
        bound = np.broadcast_to(bound, ref.shape)[ok] + u * np.abs(ref[ok])
        err = np.abs(got[ok] - ref[ok])
        assert (err <= bound).all(), (err - bound).max()
    assert np.array_equal(tt, rt)
    assert not (lp > 0).any() and not (tl > 0).any() and not (en < 0).any()
    return lp, en, tl


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("R,V", [(1, 1), (3, 1), (4, 2), (4, 100), (300, 257), (5, 2049), (2, 32000),
                                 (300, 33001), (1, 128000)])
def test_one_token_has_all(R, V, dtype):
    """One logit left, or one that is far above: its log-probability and the entropy
    are 0, not next to it."""
    g = np.random.default_rng(R + V)
    at = g.integers(0, V, R)
    for low in (-np.inf, -3.3e38, -1e4):
        x = np.full((R, V), low)
        x[np.arange(R), at] = g.choice([-5.0, 0.0, 1.0, 77.0], R)
        lp, en, tl = _check_logprobs(x, at[:, None], 1, dtype)
        assert (lp == 0).all() and (en == 0).all() and (tl == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("R,V", [(4, 60), (6, 3001), (5, 32000), (300, 32000), (3, 128000)])
def test_confident_rows(R, V, dtype):
    """The best of a row some 8 to 30 above the others: its log-probability is -(1 - p),
    with as many right digits as that has; wherever the best one stands."""
    g = np.random.default_rng(V)
    for above in (8.0, 12.5, 17.25, 30.0):
        x = g.standard_normal((R, V)) - 1.0
        at = g.integers(0, V, R)
        at[:3] = 0, V - 1, V // 2
        x[np.arange(R), at] = above
        x[0, V // 3] = above - 0.5                   # a close second
        lp, _, _ = _check_logprobs(x, np.stack([at, (at + 1) % V], 1), 3, dtype)
    assert (lp[1:, 0] > -1e-5).all() and (lp[1:, 0] < 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("R", [6, 300])
def test_references_behind_the_maximum(R, dtype):
    """Rows that rise, by steps below and above what a reference is raised for; equal
    maxima; equal rows."""
    g = np.random.default_rng(R)
    V = 40001
    at = np.arange(V)
    x = g.standard_normal((R, V))
    x[0] += 7.5 * (at >= 0.9 * V)
    x[1] += 20.0 * at / V
    x[2] += 100.0 * at / V
    x[3, V - 1], x[3, 5] = 12.0, 12.0
    x[4] = 1.5
    x[5, V - 700:] = 12.5
    for j in range(6, R):
        x[j] += (j % 17) * (at >= V - 1 - 37 * j)
    _check_logprobs(x, g.integers(0, V, (R, 2)), 4, dtype)


@pytest.mark.parametrize("dtype,Hq,Hkv,D,n,m", [
    ("bf16", 4, 2, 64, 150, 150), ("bf16", 8, 2, 128, 300, 300), ("bf16", 6, 2, 40, 700, 700),
    ("bf16", 4, 2, 128, 30, 3000), ("bf16", 4, 2, 256, 90, 900), ("bf16", 8, 2, 128, 200, 4300),
    ("bf16", 8, 2, 64, 4500, 4500), ("f32", 4, 2, 64, 150, 150), ("f32", 4, 2, 128, 200, 1500),
    ("f32", 4, 2, 64, 600, 600)])
def test_infinite_values_of_a_prompt_whatever_their_weight(dtype, Hq, Hkv, D, n, m):
    """A query that sees an infinite value gets it, NaN of a NaN or of both signs, be the
    key's weight 0, below float32 or large, wherever in its keys the key stands."""
    g = np.random.default_rng(n + D)
    q, k, v = (to_dev(draw(g, dtype, r, h, D)) for r, h in ((n, Hq), (m, Hkv), (m, Hkv)))
    q[:, :, 0], k[:, :, 0] = 1.0, 0.0
    own = m - n // 2                                 # some query's own key, and one before all
    for at in (own, 5):
        k[at, :, 0] = -INF                           # weight 0
        k[at + 1, :, 0] = -3e4                       # weight e^-3750 and less
        k[at + 2, :, 0] = 40.0
    clean, lse = ops.prompt_attention(q, k, v)
    assert torch.isfinite(clean).all()
    for at in (own, 5):
        w = v.clone()
        w[at, 0, 3], w[at + 1, 0, 4], w[at + 2, 0, 5] = INF, -INF, INF
        w[at, 1, D - 1], w[at + 1, 1, D - 1] = -INF, INF
        w[at, 1, 2] = NAN
        out, l = ops.prompt_attention(q, k, w)
        assert torch.equal(l, lse)
        token = torch.arange(n)[:, None].expand(n, Hkv) + (m - n)
        want = clean.clone()
        for h, d, key, x in ((0, 3, at, INF), (0, 4, at + 1, -INF), (0, 5, at + 2, INF),
                             (1, D - 1, at, -INF), (1, 2, at, NAN), (1, D - 1, at + 1, NAN)):
            _set(want, token[:, h] >= key, h, Hq // Hkv, d, x)
        same = (out == want) | (torch.isnan(out) & torch.isnan(want))
        assert same.all(), (at, (~same).nonzero()[:5])


def _set(want, rows, h, per, d, x):
    part = want[:, h * per:(h + 1) * per, d]
    part[rows.to(DEV)] = x


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_infinite_values_behind_keys_of_no_weight(dtype):
    # all keys of a first part of the history, which blocks of their own take
    n, m, D = 3, 5000, 64
    g = np.random.default_rng(m)
    q, k, v = (to_dev(draw(g, dtype, r, h, D)) for r, h in ((n, 4), (m, 2), (m, 2)))
    q[:, :, 0], k[:, :, 0], k[:2000, :, 0] = 1.0, 0.0, -INF
    clean, lse = ops.prompt_attention(q, k, v)
    v[20, 0, 1], v[1900, 1, 7], v[1950, 1, 7] = -INF, INF, INF
    v[4990, 0, 9] = NAN
    out, l = ops.prompt_attention(q, k, v)
    clean[:, :2, 1], clean[:, 2:, 7], clean[:, :2, 9] = -INF, INF, NAN
    same = (out == clean) | (torch.isnan(out) & torch.isnan(clean))
    assert same.all() and torch.equal(l, lse)
    k[2000:, :, 0] = -INF                            # no weight at all
    out, l = ops.prompt_attention(q, k, v)
    assert (out == 0).all() and (l == -INF).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hkv,R", [(1, 1), (4, 2), (2, 300)])
def test_nan_values_of_a_cache_of_4_bits_whatever_their_weight(Hkv, R, dtype):
    """Keys of weight 0 (scores of -inf), single ones and all of a first part, which
    blocks of their own take where rows are few: their blocks of NaN count."""
    g = np.random.default_rng(R)
    S, D = 1500, 64
    k, v = (to_dev(draw(g, "f32", S, Hkv, D)) for _ in range(2))
    k[:, :, 0] = 0.0
    k[:600, :, 0], k[1000, :, 0] = 2.0, 2.0
    cache, _ = _kv4(k, v)
    q = to_dev(draw(g, dtype, R, 2 * Hkv, D))
    q[:, :, 0] = -3e38                               # times 2 and more: -inf
    rows = torch.zeros(R, dtype=torch.int32, device=DEV)
    clean, lse = ops.kv4_attention(q, cache, cache_row=rows, scale=0.2)
    assert torch.isfinite(clean).all() and torch.isfinite(lse).all()
    for key, h, block in ((20, 0, 0), (599, Hkv - 1, 1), (1000, 0, 1), (1400, Hkv - 1, 0)):
        held = cache[3].clone()
        held[0, key, h, block] = 255
        out, l = ops.kv4_attention(q, cache[:3] + (held,), cache_row=rows, scale=0.2)
        want = clean.clone()
        want[:, 2 * h:2 * h + 2, 32 * block:32 * block + 32] = NAN
        same = (out == want) | (torch.isnan(out) & torch.isnan(want))
        assert same.all() and torch.equal(l, lse), (key, (~same).nonzero()[:4])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_small_values(dtype):
    """Values of some 2^-75 in a cache and 2^-95 in a prompt are as exact as others: terms
    of 2^-20 of them are above what may lose bits (2^-100, 2^-118)."""
    g = np.random.default_rng(8)
    S, D, n = 300, 64, 40
    k, v = draw(g, "f32", S, 1, D, std=0.3), draw(g, "f32", S, 1, D)
    q = to_dev(draw(g, dtype, n, 2, D))
    # a cache: values of some 2^-75
    cache, (kk, vv) = _kv4(to_dev(k), to_dev(v * 2.0 ** -75))
    lens = torch.arange(S - n + 1, S + 1, dtype=torch.int32, device=DEV)
    rows = torch.zeros(n, dtype=torch.int32, device=DEV)
    out, lse = ops.kv4_attention(q, cache, lens=lens, cache_row=rows, scale=0.125)
    # a prompt: of some 2^-95
    t = _dtype(dtype)
    pk, pv = to_dev(k).to(t), to_dev(v * 2.0 ** -95).to(t)
    pout, plse = ops.prompt_attention(q, pk, pv, scale=0.125)
    for got, l, k64, v64, up in ((out, lse, kk, vv, 2.0 ** 75), (pout, plse, vals(pk), vals(pv), 2.0 ** 95)):
        for r in (0, n // 2, n - 1):
            for h in range(2):
                m, x = S - n + r + 1, vals(q)[r, h]
                ref, rl = oracle.prompt.softmax_rows(0.125 * (k64[:m, 0] @ x), v64[:m, 0] * up)
                check_row(vals(got)[r, h] * up, to_host(l)[r, h], ref, rl, x, k64[:m, 0],
                          v64[:m, 0] * up, 0.125, dtype)
