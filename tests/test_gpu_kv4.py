"""moe_kv4_store, moe_kv4_load and moe_kv4_attention: codes, scales and loaded values
bit for bit against the oracle, attention within prompt_helpers.check_row (the values
of a cache are exact, so the bound is that of attention over them)."""
import numpy as np
import pytest
import torch

import oracle
from paper_2410_17954_amd import ops, synth
from gpu_helpers import to_dev, to_host, vals
from prompt_helpers import check_row, draw, values

pytestmark = pytest.mark.gpu


def _hard_blocks(g, n, Hkv, D):
    """Random values, exact ties, borders of the block's power, zeros, tiny and huge."""
    x = g.standard_normal((n, Hkv, D)) * np.exp2(g.integers(-3, 4, (n, Hkv, 1)))
    ties = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.0, -0.25, -5.0, 0.0, -0.0, 6.5])
    for i in range(0, n, 3):
        x[i] = g.choice(ties, (Hkv, D)) * 2.0 ** int(g.integers(-20, 20))
    x[1 % n, 0, :32] = 0.0
    x[2 % n, 0, :32] = g.standard_normal(32) * 2.0 ** -127
    x[4 % n, 0, :32] = g.standard_normal(32) * 2.0 ** -124
    x[5 % n, 0, :32] = 3.3e38 * np.sign(g.standard_normal(32))
    x[7 % n, 0, :32] = g.standard_normal(32) * 2.0 ** 125 / 4
    return x.astype(np.float32)


def _cast(x, dtype):
    return synth.bf16_bits(x) if dtype == "bf16" else x


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,Hkv,D", [(1, 1, 32), (13, 2, 64), (40, 3, 96), (70, 8, 128), (9, 1, 256),
                                     (12, 5, 160)])
def test_codes_scales_and_values(N, Hkv, D, dtype):
    g = np.random.default_rng(N + D)
    k, v = _cast(_hard_blocks(g, N, Hkv, D), dtype), _cast(_hard_blocks(g, N, Hkv, D), dtype)
    rows, S = 3, N // 2 + 3
    slots = g.permutation(rows * S)[:N].astype(np.int32)
    cache = tuple(t.fill_(0x5a) for t in ops.kv4_cache(rows, S, Hkv, D, "cuda:0"))
    ops.kv4_store(to_dev(k), to_dev(v), cache, slots=to_dev(slots))
    for x, codes, scales in ((k, cache[0], cache[1]), (v, cache[2], cache[3])):
        rc, rs = oracle.kv4_encode(values(x))
        codes, scales = (to_host(t).reshape(rows * S, Hkv, -1) for t in (codes, scales))
        assert np.array_equal(scales[slots], rs) and np.array_equal(codes[slots], rc)
        rest = np.setdiff1d(np.arange(rows * S), slots)     # nothing else is written
        assert (codes[rest] == 0x5a).all() and (scales[rest] == 0x5a).all()
        # half a step at most, 2^e of the block
        y = oracle.kv4_decode(rc, rs)
        top = np.abs(values(x)).reshape(N, Hkv, -1, 32).max(-1)
        ok = top <= 7 * 2.0 ** 125
        step = np.exp2(rs.astype(np.float64) - 127)
        err = np.abs(y - values(x)).reshape(N, Hkv, -1, 32).max(-1)
        assert (err <= step)[ok].all()
    for out in ("bf16", "f32"):
        t = torch.bfloat16 if out == "bf16" else torch.float32
        kk, vv = ops.kv4_load(cache, slots=to_dev(slots), dtype=t)
        for got, x in ((kk, k), (vv, v)):
            ref = oracle.kv4_decode(*oracle.kv4_encode(values(x)))
            assert got.dtype == t and np.array_equal(vals(got), ref)
            assert np.array_equal(np.signbit(vals(got)), np.signbit(ref))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_nan_blocks_and_left_out_tokens(dtype):
    g = np.random.default_rng(3)
    N, Hkv, D = 6, 2, 64
    x = g.standard_normal((N, Hkv, D)).astype(np.float32)
    x[1, 0, 5], x[2, 1, 40], x[3, 0, 63] = np.nan, np.inf, -np.inf
    k, v = _cast(x, dtype), _cast(x[::-1].copy(), dtype)
    cache = tuple(t.fill_(0x11) for t in ops.kv4_cache(2, 5, Hkv, D, "cuda:0"))
    slots = np.array([9, 0, -1, 4, 10, -2**31], np.int32)
    ops.kv4_store(to_dev(k), to_dev(v), cache, slots=to_dev(slots))
    kept = [0, 1, 3]
    for y, codes, scales in ((k, cache[0], cache[1]), (v, cache[2], cache[3])):
        rc, rs = oracle.kv4_encode(values(y))
        codes, scales = (to_host(t).reshape(10, Hkv, -1) for t in (codes, scales))
        assert np.array_equal(scales[slots[kept]], rs[kept])
        assert np.array_equal(codes[slots[kept]], rc[kept])
        rest = np.setdiff1d(np.arange(10), slots[kept])
        assert (codes[rest] == 0x11).all() and (scales[rest] == 0x11).all()
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    kk = torch.full((N, Hkv, D), 3.0, dtype=t, device="cuda:0")
    vv = kk.clone()
    ops.kv4_load(cache, slots=to_dev(slots), k=kk, v=vv)
    for got, y in ((kk, k), (vv, v)):
        ref = oracle.kv4_decode(*oracle.kv4_encode(values(y)))
        got = vals(got)
        assert np.array_equal(got[kept], ref[kept], equal_nan=True)
        assert (got[[2, 4, 5]] == 3.0).all()
    assert np.isnan(vals(kk)[1, 0, :32]).all() and not np.isnan(vals(kk)[1, 0, 32:]).any()


def test_strided_tokens_and_default_slots():
    g = np.random.default_rng(4)
    N, Hkv, D = 11, 2, 96
    buf = torch.randn(N, 7, D, device="cuda:0").bfloat16()
    k, v = buf[:, 1:3], buf[:, 4:6]
    a, b = ops.kv4_cache(1, N, Hkv, D, "cuda:0"), ops.kv4_cache(1, N, Hkv, D, "cuda:0")
    ops.kv4_store(k, v, a)
    ops.kv4_store(k.contiguous(), v.contiguous(), b)
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    keep = buf.clone()
    ops.kv4_load(a, k=buf[:, 0:2], v=buf[:, 5:7])
    kk, vv = ops.kv4_load(a)
    assert torch.equal(buf[:, 0:2], kk) and torch.equal(buf[:, 5:7], vv)
    assert torch.equal(buf[:, 2:5], keep[:, 2:5])


def _cache_of(g, C, S, Hkv, D):
    x = [g.standard_normal((C, S, Hkv, D)) for _ in range(2)]
    host = []
    for y in x:
        host += list(_encode_fast(y))
    return host, tuple(to_dev(a) for a in host)


def _encode_fast(x):
    """oracle.kv4_encode over whole arrays (its pins: test_prompt_host)."""
    y = x.reshape(x.shape[:-1] + (-1, 32))
    top = np.abs(y).max(-1)
    e = np.clip(np.ceil(np.log2(top / 7)), -124, 125)
    q = np.abs(y) / np.exp2(e)[..., None]
    c = np.abs(q[..., None] - oracle.prompt.E2M1).argmin(-1).astype(np.uint8)
    c = (c | np.signbit(y).astype(np.uint8) << 3).reshape(x.shape)
    return c[..., 0::2] | c[..., 1::2] << 4, (e + 127).astype(np.uint8)


def _attend(g, dtype, C, S, Hq, Hkv, D, rows, lens, scale, std=2.0, poison=True):
    host, cache = _cache_of(g, C, S, Hkv, D)
    R = len(rows)
    q = draw(g, dtype, R, Hq, D, std=std)
    rows, lens = np.asarray(rows, np.int32), np.asarray(lens, np.int32)
    n = np.clip(lens, 0, S)
    if poison:                          # what no row reads is NaN
        for c in range(C):
            end = max([n[r] for r in range(R) if rows[r] == c], default=0)
            for t in (cache[1], cache[3]):
                t[c, end:] = 255
    out, lse = ops.kv4_attention(to_dev(q), cache, lens=to_dev(lens), cache_row=to_dev(rows),
                                 scale=scale)
    o, l = vals(out), to_host(lse).astype(np.float64)
    for r in range(R):
        if not 0 <= rows[r] < C:
            assert (o[r] == 0).all() and (l[r] == -np.inf).all()
            continue
        k, v = (oracle.kv4_decode(host[2 * j][rows[r], :n[r]], host[2 * j + 1][rows[r], :n[r]])
                for j in range(2))
        for h in range(Hq):
            kk, vv = k[:, h // (Hq // Hkv)], v[:, h // (Hq // Hkv)]
            x = values(q)[r, h]
            ref, rl = oracle.prompt.softmax_rows(scale * (kk @ x), vv)
            check_row(o[r, h], l[r, h], ref, rl, x, kk, vv, scale, dtype)
    return out, lse, q, cache


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv,D", [(4, 4, 64), (8, 2, 128), (6, 2, 32), (16, 1, 96), (3, 3, 256),
                                      (40, 2, 128), (34, 1, 64), (4, 2, 160), (2, 1, 224),
                                      (7, 7, 192)])
def test_attention_heads_and_dimensions(Hq, Hkv, D, dtype):
    g = np.random.default_rng(D + Hq)
    _attend(g, dtype, 4, 150, Hq, Hkv, D, [2, 0, 3, 1, 0], [150, 77, 1, 0, 33], D ** -0.5)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("S", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 257, 1000,
                               4100])
def test_attention_lengths(S, dtype):
    g = np.random.default_rng(S)
    _attend(g, dtype, 3, S, 4, 2, 64, [0, 1, 2, 1, 7, -1], [S, S - 1, (S + 1) // 2, S + 5, S, S], 0.2)


def test_attention_defaults_and_workspace():
    g = np.random.default_rng(5)
    _, cache = _cache_of(g, 3, 70, 2, 64)
    q = to_dev(draw(g, "bf16", 3, 8, 64))
    rows = torch.arange(3, dtype=torch.int32, device="cuda:0")
    lens = torch.full((3,), 70, dtype=torch.int32, device="cuda:0")
    a = ops.kv4_attention(q, cache)
    ws = ops.workspace_tensor(max(1, ops.kv4_attention_workspace(3, 70, 8, 2, 64)), "cuda:0")
    b = ops.kv4_attention(q, cache, lens=lens, cache_row=rows, scale=64 ** -0.5, workspace=ws)
    c = ops.kv4_attention(q, cache, want_lse=False)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    assert torch.equal(a[0], c[0]) and c[1] is None


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_nan_blocks_scales_and_signs(dtype):
    g = np.random.default_rng(6)
    out, lse, q, cache = _attend(g, dtype, 2, 90, 4, 2, 128, [0, 1], [90, 50], -0.1)
    _attend(g, dtype, 2, 90, 4, 2, 128, [0, 1], [90, 50], 0.0)
    cache[3][0, 17, 1, 2] = 255                      # one block of values of head 1
    o2, l2 = ops.kv4_attention(to_dev(q), cache, lens=torch.tensor([90, 50], dtype=torch.int32,
                                                                   device="cuda:0"), scale=-0.1)
    assert torch.isnan(o2[0, 2:, 64:96]).all()
    o2[0, 2:, 64:96] = out[0, 2:, 64:96]
    assert torch.equal(o2, out) and torch.equal(l2, lse)
    cache[1][1, 3, 0, 0] = 255                       # one block of keys of head 0
    o2, l2 = ops.kv4_attention(to_dev(q), cache, lens=torch.tensor([90, 50], dtype=torch.int32,
                                                                   device="cuda:0"), scale=-0.1)
    assert torch.isnan(o2[1, :2]).all() and torch.isnan(l2[1, :2]).all()
    assert torch.equal(o2[1, 2:], out[1, 2:]) and torch.equal(l2[0], lse[0])


def test_attention_cache_past_32_bits():
    # the last row's codes lie beyond 2^32 bytes
    C, S, Hkv, D = 2, 1 << 21, 20, 128
    cache = tuple(torch.zeros((C, S, Hkv, w), dtype=torch.uint8, device="cuda:0")
                  for w in (D // 2, D // 32) * 2)
    g = torch.Generator(device="cuda:0")
    g.manual_seed(1)
    n = 2000
    k = torch.randn(n, Hkv, D, device="cuda:0", generator=g)
    v = torch.randn(n, Hkv, D, device="cuda:0", generator=g)
    slots = (C * S - n + torch.arange(n, device="cuda:0")).int()
    assert int(slots[0]) * Hkv * (D // 2) > 2 ** 32
    ops.kv4_store(k, v, cache, slots=slots)
    kk, vv = ops.kv4_load(cache, slots=slots)
    q = torch.randn(1, Hkv, D, device="cuda:0", generator=g).bfloat16()
    row = torch.tensor([1], dtype=torch.int32, device="cuda:0")
    # keys before them are zeros: their scores are 0, their values 0
    out, lse = ops.kv4_attention(q, cache, cache_row=row)
    s = torch.einsum("hd,nhd->hn", q[0].double().cpu(), kk.double().cpu()) * D ** -0.5
    p = s.exp()
    total = p.sum(1) + (S - n)
    ref = torch.einsum("hn,nhd->hd", p, vv.double().cpu()) / total[:, None]
    # weights sum to 1; numerators of bf16 2^-8, sums of S / 64 terms and more 2^-9
    bound = (p[..., None] * vv.double().cpu().abs().permute(1, 0, 2)).sum(1) / total[:, None] * 2 ** -6
    assert ((out[0].double().cpu() - ref).abs() <= bound).all()
    assert (lse[0].double().cpu() - total.log()).abs().max() <= 2 ** -6


@pytest.mark.parametrize("S", [50, 700])
def test_attention_of_scores_that_are_all_minus_infinity(S):
    # an infinite query against keys of one sign: no weight, whatever the values hold
    cache = ops.kv4_cache(1, S, 1, 64, "cuda:0")
    k = torch.zeros((S, 1, 64), device="cuda:0")
    k[:, :, 0] = 1.0
    ops.kv4_store(k, torch.randn_like(k), cache)
    cache[3][:, ::5] = 255
    q = torch.zeros((1, 2, 64), device="cuda:0")
    q[:, 0, 0] = -3e38                               # times 1e3: -inf
    out, lse = ops.kv4_attention(q.bfloat16(), cache, scale=1e3)
    assert (out[0, 0] == 0).all() and lse[0, 0] == -float("inf")
    assert torch.isnan(out[0, 1]).all() and abs(float(lse[0, 1]) - np.log(S)) < 1e-5
