"""moe_prompt_attention against the float64 oracle, within the bound of
prompt_helpers.check_row."""
import numpy as np
import pytest
import torch

import oracle
from paper_2410_17954_amd import ops
from gpu_helpers import to_dev, to_host, vals
from prompt_helpers import check_row, draw, values

pytestmark = pytest.mark.gpu


def _case(dtype, nq, nk, Hq, Hkv, D, seed, before=0, after=0):
    """Sequences of nq[b] queries over nk[b] keys; `before` and `after` rows of q
    belong to none."""
    g = np.random.default_rng(seed)
    qo = before + np.concatenate([[0], np.cumsum(nq)])
    ko = np.concatenate([[0], np.cumsum(nk)])
    return dict(q=draw(g, dtype, int(qo[-1]) + after, Hq, D, std=2.0),
                k=draw(g, dtype, int(ko[-1]), Hkv, D), v=draw(g, dtype, int(ko[-1]), Hkv, D),
                qo=qo.astype(np.int32), ko=ko.astype(np.int32)), g


def _check(c, dtype, scale, rows=None, strided=False, plain_offsets=False, **kw):
    d = {n: to_dev(a) for n, a in c.items()}
    if strided:                        # a fused projection: tokens of q, k and v side by side
        N, M = len(c["q"]), len(c["k"])
        Hq, D = c["q"].shape[1:]
        Hkv = c["k"].shape[1]
        buf = torch.full((max(N, M), Hq + 2 * Hkv + 3, D), float("nan"), dtype=d["q"].dtype,
                         device="cuda:0")
        at = 1
        for n, heads in (("q", Hq), ("k", Hkv), ("v", Hkv)):
            buf[:len(d[n]), at:at + heads] = d[n]
            d[n] = buf[:len(d[n]), at:at + heads]
            at += heads
    N, Hq, D = c["q"].shape
    out = torch.full((N, Hq, D), 7.0, dtype=d["q"].dtype, device="cuda:0")
    lse = torch.full((N, Hq), 9.0, device="cuda:0")
    got = ops.prompt_attention(d["q"], d["k"], d["v"],
                               q_offsets=None if plain_offsets else d["qo"],
                               k_offsets=None if plain_offsets else d["ko"], scale=scale, out=out,
                               lse=lse, **kw)
    assert got[0] is out and got[1] is lse
    q, k, v = (values(c[n]) for n in ("q", "k", "v"))
    o, l = vals(out), to_host(lse).astype(np.float64)
    n_q = Hq // k.shape[1]
    member = np.zeros(N, bool)
    for b in range(len(c["qo"]) - 1):
        n, m = c["qo"][b + 1] - c["qo"][b], c["ko"][b + 1] - c["ko"][b]
        for i in range(n):
            r = c["qo"][b] + i
            member[r] = True
            if rows is not None and r not in rows:
                continue
            keys = slice(c["ko"][b], c["ko"][b] + max(0, m - n + i + 1))
            for h in range(Hq):
                kk, vv = k[keys, h // n_q], v[keys, h // n_q]
                ref, rl = oracle.prompt.softmax_rows(scale * (kk @ q[r, h]), vv)
                check_row(o[r, h], l[r, h], ref, rl, q[r, h], kk, vv, scale, dtype)
    assert (o[~member] == 7.0).all() and (l[~member] == 9.0).all()
    return out, lse


DIMS = [(4, 4, 64), (8, 2, 128), (6, 2, 40), (16, 1, 80), (3, 3, 256), (40, 2, 128), (2, 1, 8),
        (4, 2, 200), (5, 1, 32), (33, 1, 72)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv,D", DIMS)
def test_heads_and_dimensions(Hq, Hkv, D, dtype):
    c, _ = _case(dtype, [5, 70, 1, 33], [5, 70, 20, 40], Hq, Hkv, D, D + Hq)
    _check(c, dtype, D ** -0.5)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,m", [(1, 1), (2, 2), (31, 31), (32, 32), (33, 33), (63, 64), (64, 64),
                                 (65, 65), (127, 128), (128, 128), (129, 129), (257, 257), (1, 1000),
                                 (3, 4097), (200, 231), (40, 33), (7, 0), (513, 513)])
def test_lengths(n, m, dtype):
    c, _ = _case(dtype, [n], [m], 4, 2, 64, n * 7 + m)
    _check(c, dtype, 0.2)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128, 192])
def test_packed_sequences(D, dtype):
    # empty ones, ones without keys, ones longer in keys, rows of no sequence
    c, _ = _case(dtype, [0, 3, 100, 0, 1, 65, 17, 5, 0], [0, 3, 100, 9, 1, 300, 0, 4, 2], 6, 2, D,
                 D, before=2, after=3)
    _check(c, dtype, 0.1)
    assert c["qo"][0] == 2


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strided_tokens_and_default_offsets(dtype):
    c, _ = _case(dtype, [50, 30], [50, 30], 8, 2, 64, 5)
    _check(c, dtype, 0.125, strided=True)
    c, _ = _case(dtype, [70], [70], 8, 2, 64, 6)
    _check(c, dtype, 0.125, plain_offsets=True)
    d = {n: to_dev(a) for n, a in c.items()}
    a = ops.prompt_attention(d["q"], d["k"], d["v"])
    b = ops.prompt_attention(d["q"], d["k"], d["v"], q_offsets=d["qo"], want_lse=False)
    assert torch.equal(a[0], b[0]) and b[1] is None


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_what_later_tokens_hold_stays_out(D, dtype):
    # a NaN or infinity in a key or value reaches its own query and those after it
    n = 150
    c, g = _case(dtype, [n], [n], 4, 2, D, 3)
    clean = ops.prompt_attention(*(to_dev(c[x]) for x in ("q", "k", "v")))
    k, v = (to_dev(c[x]) for x in ("k", "v"))
    v[40, 0, 3], v[97, 1, D - 1], v[149, 0, 0] = float("nan"), float("inf"), float("-inf")
    k[130, 0, 1] = float("nan")
    out, lse = ops.prompt_attention(to_dev(c["q"]), k, v)
    torch.cuda.synchronize()
    same = (out == clean[0])
    assert same[:40].all() and same[:97, 2:].all()
    assert torch.isnan(out[40:, :2, 3]).all() and same[40:130, :2, 4:].all()
    assert (out[97:, 2:, D - 1] == float("inf")).all() and same[97:, 2:, :D - 1].all()
    assert torch.isnan(out[130:, :2]).all() and torch.isnan(lse[130:, :2]).all()
    assert torch.equal(lse[:130], clean[1][:130]) and torch.equal(lse[:, 2:], clean[1][:, 2:])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scores_of_minus_infinity_and_extreme_scales(dtype):
    n, D = 70, 64
    c, _ = _case(dtype, [n], [n], 2, 1, D, 8)
    q, k, v = (to_dev(c[x]) for x in ("q", "k", "v"))
    q[:, :, 0], k[:, :, 0] = 1.0, 0.0
    k[:20, :, 0] = float("-inf")                     # nothing before token 20
    out, lse = ops.prompt_attention(q, k, v)
    assert (out[:20] == 0).all() and (lse[:20] == -float("inf")).all()
    ref = ops.prompt_attention(q[20:], k[20:], v[20:])
    tol = 2.0 ** -7 if dtype == "bf16" else 2.0 ** -20
    # of one set of keys, in tiles that begin elsewhere: roundings of numerators and of
    # the result, relative to values of at most 5
    assert (out[20:].float() - ref[0].float()).abs().max() <= 5 * 2 * tol
    out, lse = ops.prompt_attention(q[20:], k[20:], v[20:], scale=0.0)
    m = v[20:].float().cumsum(0) / torch.arange(1, n - 19, device="cuda:0")[:, None, None]
    assert (out.float() - m).abs().max() <= 5 * tol
    assert (lse - torch.arange(1, n - 19, device="cuda:0").float().log()[:, None]).abs().max() <= 1e-5
    c, _ = _case(dtype, [n], [n], 2, 1, D, 9)
    _check(c, dtype, -0.125)


def test_many_sequences_of_one_token():
    c, _ = _case("bf16", [1] * 300, [1 + (i * 37) % 90 for i in range(300)], 8, 2, 64, 12)
    _check(c, "bf16", 0.125)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_few_queries_behind_many_keys(dtype):
    # keys are split over blocks and joined
    c, _ = _case(dtype, [3, 40], [5000, 3000], 4, 1, 128, 21)
    a = _check(c, dtype, 0.09)
    b = _check(c, dtype, 0.09)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_long_prompt_and_repeatability():
    c, _ = _case("bf16", [2500, 100], [2500, 1300], 4, 2, 128, 31)
    rows = set(list(range(0, 40)) + list(range(1000, 1070, 7)) + list(range(2440, 2600, 5)))
    a = _check(c, "bf16", 0.088, rows=rows)
    b = _check(c, "bf16", 0.088, rows={0})
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_offsets_past_32_bits():
    # tokens 2^23 elements apart: the last key lies beyond 2^32 bytes
    n, Hq, Hkv, D, stride = 300, 2, 1, 64, 1 << 23
    c, _ = _case("bf16", [n], [n], Hq, Hkv, D, 41)
    buf = torch.empty(n * stride, dtype=torch.bfloat16, device="cuda:0")
    view = lambda at, h: buf.as_strided((n, h, D), (stride, D, 1), at)
    for name, at, h in (("q", 0, Hq), ("k", Hq * D, Hkv), ("v", (Hq + Hkv) * D, Hkv)):
        view(at, h).copy_(to_dev(c[name]))
    q, k, v = view(0, Hq), view(Hq * D, Hkv), view((Hq + Hkv) * D, Hkv)
    got = ops.prompt_attention(q, k, v)
    ref = ops.prompt_attention(*(to_dev(c[x]) for x in ("q", "k", "v")))
    assert torch.equal(got[0], ref[0]) and torch.equal(got[1], ref[1])


@pytest.mark.parametrize("dtype,Hq,Hkv,D,n,m", [
    ("bf16", 8, 2, 128, 300, 5000),      # blocks of eight waves, keys split
    ("bf16", 4, 1, 64, 200, 4200), ("bf16", 8, 2, 256, 70, 4500), ("bf16", 6, 2, 80, 130, 4300),
    ("bf16", 8, 2, 128, 90, 700),        # two groups of waves
    ("bf16", 3, 3, 256, 60, 600), ("bf16", 7, 1, 40, 33, 520), ("f32", 4, 2, 64, 50, 600),
    ("f32", 4, 2, 128, 50, 600)])
def test_every_kind_of_block(dtype, Hq, Hkv, D, n, m):
    c, g = _case(dtype, [n, 3, 0, 40], [m, m + 9, 5, m - 100], Hq, Hkv, D, n + m + D)
    rows = set(range(0, 12)) | set(range(n - 9, n + 14)) | {n // 2, n + 42}
    _check(c, dtype, D ** -0.5, rows=rows)
    # a value that is no number is seen from its token on
    v = to_dev(c["v"])
    at = m - n // 2
    v[at, 0, D - 3] = float("nan")
    out, _ = ops.prompt_attention(to_dev(c["q"]), to_dev(c["k"]), v, q_offsets=to_dev(c["qo"]),
                                  k_offsets=to_dev(c["ko"]))
    first = at - (m - n)
    bad = torch.isnan(out)
    assert bad[first:n, :Hq // Hkv, D - 3].all() and bad.sum() == (n - first) * (Hq // Hkv)


@pytest.mark.parametrize("dtype,Hq,Hkv,D,nq,nk", [
    ("bf16", 8, 2, 128, [300], [300]),                     # four groups of waves
    ("bf16", 8, 2, 64, [260, 1, 0], [1500, 400, 7]), ("bf16", 16, 2, 96, [257, 33], [257, 300]),
    ("bf16", 4, 1, 40, [70], [2100]), ("bf16", 7, 1, 128, [64], [1100]),   # and splits
    ("bf16", 32, 8, 128, [600], [600]),                    # two
    ("bf16", 6, 2, 256, [100], [900]), ("bf16", 4, 1, 128, [20], [900]),
    ("f32", 4, 2, 64, [100, 30], [900, 700])])
def test_groups_of_waves(dtype, Hq, Hkv, D, nq, nk):
    c, g = _case(dtype, nq, nk, Hq, Hkv, D, sum(nk) + D)
    N = sum(nq)
    rows = set(range(0, 5)) | set(range(nq[0] - 5, nq[0] + 3)) | {nq[0] // 2, N - 1}
    a = _check(c, dtype, D ** -0.5, rows=rows)
    b = _check(c, dtype, D ** -0.5, rows={0})
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    v = to_dev(c["v"])
    at = nk[0] - nq[0] // 2            # a value that is no number is seen from its token on
    v[at, Hkv - 1, D - 1], first = float("inf"), at - (nk[0] - nq[0])
    out, _ = ops.prompt_attention(to_dev(c["q"]), to_dev(c["k"]), v, q_offsets=to_dev(c["qo"]),
                                  k_offsets=to_dev(c["ko"]))
    bad = out == float("inf")
    assert bad[first:nq[0], -(Hq // Hkv):, D - 1].all()
    assert bad.sum() == (nq[0] - first) * (Hq // Hkv) and torch.isfinite(out[~bad]).all()


def test_more_sequences_than_tiles():
    # most of them empty; the others' keys would be split over blocks
    c, g = _case("bf16", [1, 2], [3000, 2000], 4, 1, 64, 77)
    B = 70000
    qo, ko = np.zeros(B + 1, np.int32), np.zeros(B + 1, np.int32)
    qo[30000:], ko[30000:] = 1, 3000
    qo[69000:], ko[69000:] = 3, 5000
    got = ops.prompt_attention(*(to_dev(c[n]) for n in ("q", "k", "v")), q_offsets=to_dev(qo),
                               k_offsets=to_dev(ko))
    ref = ops.prompt_attention(*(to_dev(c[n]) for n in ("q", "k", "v")), q_offsets=to_dev(c["qo"]),
                               k_offsets=to_dev(c["ko"]))
    # in other splits: roundings of numerators and results of at most 1
    assert (got[0].float() - ref[0].float()).abs().max() <= 2.0 ** -7
    assert (got[1] - ref[1]).abs().max() <= 2.0 ** -14


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,m", [(70, 70), (40, 900), (3, 3000)])
def test_no_weight_whatever_the_values_hold(n, m, dtype):
    c, _ = _case(dtype, [n], [m], 4, 2, 64, n)
    q, k, v = (to_dev(c[x]) for x in ("q", "k", "v"))
    q[:, :, 0], k[:, :, 0] = 1.0, float("-inf")
    v[::3, 0, 5], v[::7, 1, 6], v[m - 1, 0, 7] = float("nan"), float("inf"), float("nan")
    out, lse = ops.prompt_attention(q, k, v)
    assert (out == 0).all() and (lse == -float("inf")).all()
