"""moe_prefix_attention against the float64 oracle, within bounds from the
roundings. With weights w_i = softmax(s)_i over N keys:
* a score is a float32 sum of D products, times scale log2 e: off by at most
  e_i = 2 (D + 1) 2^-24 |scale| sum |q k| + 3 2^-24 |s_i| (the factor 2: the
  additions of the matrix cores may round either way), and the exponential of
  the difference to the running maximum by (|s_i - max| + 3) 2^-23 more, also
  where a later maximum rescales it; together eps_i, relative to w_i;
* the numerators are rounded to the type for the second product: u (2^-8 bf16,
  nothing for float32); sums of at most N / 16 + 40 terms in a row (a lane adds
  up a sixteenth of a wave's keys, then lanes, waves, splits): c = that many
  2^-23;
* out is rounded once: u |out| (2^-24 float32).
|d out| <= sum w_i |v_i| (u + eps_i + c) + |out| (sum w_i eps_i + c) + u |out|,
|d lse| <= sum w_i eps_i + c + 2^-22 |lse|."""
import numpy as np
import pytest
import torch

import oracle
from paper_2410_17954_amd import ops, synth
from gpu_helpers import to_dev, to_host, vals

pytestmark = pytest.mark.gpu


def _case(dtype, offsets, R, Hq, Hkv, D, P, S, seed, qstd=2.0):
    g = np.random.default_rng(seed)
    G = len(offsets) - 1

    def draw(*shape, std=1.0):
        a = (std * g.standard_normal(shape)).astype(np.float32)
        return synth.bf16_bits(a) if dtype == "bf16" else a

    return dict(q=draw(R, Hq, D, std=qstd), kp=draw(G, P, Hkv, D), vp=draw(G, P, Hkv, D),
                ks=draw(R, S, Hkv, D), vs=draw(R, S, Hkv, D),
                pl=g.integers(0, P + 1, size=G).astype(np.int32),
                sl=g.integers(0, S + 1, size=R).astype(np.int32),
                off=np.asarray(offsets, np.int32)), g


def _f(a):
    return synth.values(a) if a.dtype == np.uint16 else a.astype(np.float64)


def _check(c, dtype, scale, even=False, dev=None, **kw):
    d = {n: to_dev(a) for n, a in c.items()} if dev is None else dev
    R, Hq, D = c["q"].shape
    has_p, has_s = c["kp"].shape[1] > 0, c["ks"].shape[1] > 0
    out = torch.full((R, Hq, D), 7.0, dtype=d["q"].dtype, device="cuda:0")
    lse = torch.full((R, Hq), 9.0, device="cuda:0")
    got = ops.prefix_attention(
        d["q"], d["kp"] if has_p else None, d["vp"] if has_p else None,
        d["ks"] if has_s else None, d["vs"] if has_s else None,
        prefix_len=d["pl"] if has_p else None, suffix_len=d["sl"],
        group_offsets=None if even else d["off"], scale=scale, out=out, lse=lse, **kw)
    assert got[0] is out and got[1] is lse
    q, kp, vp, ks, vs = (_f(c[n]) for n in ("q", "kp", "vp", "ks", "vs"))
    P, S = kp.shape[1], ks.shape[1]
    pl = np.clip(c["pl"], 0, P)
    sl = np.clip(c["sl"], 0, S)
    off = np.clip(c["off"], 0, R)
    ro, rl = oracle.prefix_attention(q, kp, vp, pl, ks, vs, sl, off, scale,
                                     np.full((R, Hq, D), 7.0), np.full((R, Hq), 9.0))
    o, l = vals(out), to_host(lse).astype(np.float64)
    u = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    worst = 0.0
    n_q = Hq // kp.shape[2]
    member = np.zeros(R, bool)
    for g in range(len(off) - 1):
        for r in range(off[g], off[g + 1]):
            member[r] = True
            for h in range(Hq):
                k = np.concatenate([kp[g, :pl[g], h // n_q], ks[r, :sl[r], h // n_q]])
                v = np.concatenate([vp[g, :pl[g], h // n_q], vs[r, :sl[r], h // n_q]])
                if len(k) == 0:
                    assert (o[r, h] == 0).all() and l[r, h] == -np.inf
                    continue
                s = scale * (k @ q[r, h])
                e = 2 * (D + 1) * 2.0 ** -24 * abs(scale) * (np.abs(k) @ np.abs(q[r, h]))
                eps = e + 3 * 2.0 ** -24 * np.abs(s) + (s.max() - s + 3) * 2.0 ** -23
                w = np.exp(s - rl[r, h])
                cc = (len(k) / 16 + 40) * 2.0 ** -23
                we = w @ eps + cc
                un = u if dtype == "bf16" else 0.0
                bound = (w * (un + eps + cc)) @ np.abs(v) + np.abs(ro[r, h]) * (we + u) + 1e-37
                bound *= 1 + u
                err = np.abs(o[r, h] - ro[r, h])
                assert (err <= bound).all(), (r, h, (err / bound).max())
                assert abs(l[r, h] - rl[r, h]) <= we + 2.0 ** -22 * abs(rl[r, h])
                worst = max(worst, (err / bound).max())
    # rows of no group are left as they were
    assert (o[~member] == 7.0).all() and (l[~member] == 9.0).all()
    return out, lse, worst


DIMS = [(4, 4, 64), (8, 2, 128), (6, 2, 40), (16, 1, 80), (3, 3, 256), (40, 2, 128), (2, 1, 8),
        (4, 2, 200)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv,D", DIMS)
def test_heads_and_dimensions(Hq, Hkv, D, dtype):
    c, _ = _case(dtype, [0, 3, 4, 9], 9, Hq, Hkv, D, 70, 37, D + Hq)
    _check(c, dtype, D ** -0.5)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("P,S", [(1, 1), (0, 5), (31, 0), (32, 32), (33, 31), (127, 129), (1000, 3),
                                 (4, 700)])
def test_lengths(P, S, dtype):
    c, _ = _case(dtype, [0, 2, 2, 6], 6, 4, 2, 64, P, S, P * 7 + S)
    _check(c, dtype, 0.2)
    c["pl"][:], c["sl"][:] = P, S                    # everything
    _check(c, dtype, 0.2)
    c["pl"][:], c["sl"][:] = 0, 0                    # no key at all
    _check(c, dtype, 0.2)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv,D", DIMS)
def test_heads_and_dimensions_of_longer_caches(Hq, Hkv, D, dtype):
    # more keys than one block takes for a row: splits and their join
    c, _ = _case(dtype, [0, 3, 4, 9], 9, Hq, Hkv, D, 570, 37, D + Hq)
    _check(c, dtype, D ** -0.5)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("S", [19, 540])
def test_few_keys_of_the_capacity(S, dtype):
    # the same lengths, from none to a few steps, in caches whose capacity is short
    # (a block a row) and long (splits, most without a key)
    c, _ = _case(dtype, [0, 1, 2, 4, 5, 9, 12], 12, 4, 2, 64, 160, S, 3)
    c["pl"][:] = [0, 1, 15, 31, 33, 100]
    c["sl"][:] = [0, 1, 16, 17, 5, 0, 19, 2, 18, 1, 0, 8]
    _check(c, dtype, 0.2)


@pytest.mark.parametrize("P,S", [(512, 0), (511, 1), (480, 32), (513, 0), (481, 32), (0, 512),
                                 (256, 0), (225, 31)])
def test_capacities_about_the_limit_of_one_block(P, S):
    for dtype, D in (("bf16", 64), ("bf16", 256), ("f32", 64)):
        c, _ = _case(dtype, [0, 2, 3], 3, 2, 1, D, P, S, P + S)
        _check(c, dtype, 0.1)
        c["pl"][:], c["sl"][:] = P, S
        _check(c, dtype, 0.1)


@pytest.mark.parametrize("rows,Hq,Hkv", [(1, 2, 2), (9, 2, 1), (17, 8, 2), (64, 4, 1), (130, 2, 1)])
def test_shared_by_many_rows(rows, Hq, Hkv):
    # one to seventeen tiles of sixteen query columns behind one prefix
    c, _ = _case("bf16", [0, rows], rows, Hq, Hkv, 128, 333, 20, rows)
    _check(c, "bf16", 0.09, even=True)


@pytest.mark.parametrize("rows,P,D", [(33, 1, 128), (17, 63, 64), (40, 64, 128), (70, 65, 40),
                                      (70, 31, 128), (35, 97, 104), (100, 700, 64)])
def test_shared_by_more_rows_than_a_block_has(rows, P, D):
    # more than 64 and more than 128 columns: whole and cut steps, lengths that leave
    # parts without a key, a group of few rows beside the large one
    c, g = _case("bf16", [0, rows, rows + 1, rows + 3], rows + 5, 8, 2, D, P, 9, rows + P)
    c["pl"][0] = P
    _check(c, "bf16", D ** -0.5)
    _check(c, "bf16", -0.3)
    c["pl"][:] = 0
    _check(c, "bf16", 0.1)


@pytest.mark.parametrize("rows", [5, 40])
def test_scale_of_zero_is_the_mean(rows):
    # scores of 1e36 times 0: equal weights, masked keys none
    c, g = _case("bf16", [0, rows, rows + 2], rows + 2, 8, 2, 64, 45, 6, 9)
    c["pl"][0] = 37
    for n in ("q", "kp", "ks"):
        c[n] = synth.bf16_bits((_f(c[n]) * 1e17).astype(np.float32))
    _check(c, "bf16", 0.0)
    _check(c, "bf16", -0.0)


def test_groups_rows_outside_and_bad_numbers():
    # rows before the first group and behind the last keep their outputs; lengths
    # and offsets outside their range are clipped
    c, _ = _case("bf16", [2, 2, 7, 7, 8], 11, 4, 2, 64, 50, 9, 1)
    c["pl"][:] = [9, -3, 5, 1000]
    c["sl"][3], c["sl"][4] = -1, 77
    _check(c, "bf16", 0.125)
    c["off"] = np.array([-4, 1, 5, 5, 40], np.int32)
    _check(c, "bf16", 0.125)


def test_nothing_is_taken_from_past_a_length():
    c, g = _case("bf16", [0, 4, 8], 8, 8, 2, 128, 200, 60, 6)
    c["pl"][:] = [77, 0]
    c["sl"][:] = [0, 1, 31, 32, 33, 59, 60, 0]
    clean = _check(c, "bf16", 0.09)
    for fill in (0x7fc0, 0x7f80, 0xff80, 0x7f7f):     # NaN, +inf, -inf, the largest number
        for n in ("kp", "vp"):
            for gi in range(2):
                c[n][gi, c["pl"][gi]:] = fill
        for n in ("ks", "vs"):
            for r in range(8):
                c[n][r, c["sl"][r]:] = fill
        d = {n: to_dev(a) for n, a in c.items()}
        ws = ops.workspace_tensor(ops.prefix_attention_workspace(8, 2, 8, 2, 128, 200, 60), "cuda:0")
        ws.fill_(255)
        out, lse = ops.prefix_attention(d["q"], d["kp"], d["vp"], d["ks"], d["vs"],
                                        prefix_len=d["pl"], suffix_len=d["sl"],
                                        group_offsets=d["off"], scale=0.09, workspace=ws)
        assert torch.equal(out, clean[0]) and torch.equal(lse, clean[1])


def test_large_and_equal_scores():
    c, _ = _case("f32", [0, 3], 3, 2, 1, 64, 300, 10, 9, qstd=60.0)
    c["pl"][:], c["sl"][:] = 300, 10
    _check(c, "f32", 1.0)                             # scores of some hundreds
    _check(c, "f32", -0.5)                            # a negative scale
    _check(c, "f32", 0.0)                             # all equal: the mean
    c["q"][:] = 0
    out, lse, _ = _check(c, "f32", 1.0)
    assert np.allclose(to_host(lse), np.log(310.0), rtol=1e-6)


def test_infinite_scores():
    # a key of -inf in one dimension gets no weight; where all do, IEEE gives NaN
    c, _ = _case("f32", [0, 2], 2, 1, 1, 8, 40, 0, 3)
    c["pl"][:] = 40
    c["q"][:, :, 0] = 1.0
    c["kp"][0, 1::2, 0, 0] = -np.inf
    d = {n: to_dev(a) for n, a in c.items()}
    out, lse = ops.prefix_attention(d["q"], d["kp"], d["vp"], scale=0.3)
    half = dict(c, kp=c["kp"][:, ::2].copy(), vp=c["vp"][:, ::2].copy(), pl=np.array([20], np.int32))
    ro, rl = oracle.prefix_attention(half["q"], half["kp"].astype(np.float64),
                                     half["vp"].astype(np.float64), [20], c["ks"], c["vs"], [0, 0],
                                     [0, 2], 0.3)
    assert np.abs(to_host(out) - ro).max() < 1e-5 and np.abs(to_host(lse) - rl).max() < 1e-5


def test_long_shared_prefix_and_64_bit_offsets():
    # the last group's prefix begins past 4 GiB of keys
    G, P, Hkv, D, R = 3, 1 << 20, 8, 128, 6
    kp = torch.zeros((G, P, Hkv, D), dtype=torch.bfloat16, device="cuda:0")
    vp = torch.zeros_like(kp)
    gen = torch.Generator(device="cuda:0").manual_seed(5)
    q = torch.randn((R, Hkv, D), device="cuda:0", generator=gen).bfloat16()
    # value dimension 0 counts positions: exact means, scale 0
    pos = (torch.arange(P, device="cuda:0") % 256).bfloat16()
    vp[..., 0] = pos[None, :, None]
    vp[2, P - 256:, :, 1] = 2048.0
    out, lse = ops.prefix_attention(q, kp, vp, scale=0.0)
    assert torch.equal(out[..., 0], torch.full_like(out[..., 0], 127.5))
    assert torch.equal(out[4:, :, 1], torch.full_like(out[4:, :, 1], 0.5))
    assert float(out[:4, :, 1].abs().max()) == 0.0
    assert (lse - np.log(P)).abs().max() < 1e-4
    # and by weight: only the last key of the last group scores
    kp[2, P - 1] = q[4] * 4
    o2, _ = ops.prefix_attention(q, kp, vp, scale=1.0)
    assert (o2[4, :, 1] > 2000).all() and (o2[4, :, 0] > 250).all()


@pytest.mark.parametrize("B,K", [(2, 4), (5, 3)])
def test_prefix_equals_copies_in_every_row(B, K):
    """The prefix read once for a request's beams against the same keys copied
    into every beam's suffix: the same attention within the type's rounding."""
    R, Hq, Hkv, D, P, S = B * K, 16, 4, 128, 260, 30
    c, g = _case("bf16", list(range(0, R + 1, K)), R, Hq, Hkv, D, P, S, B)
    c["pl"][:] = P
    c["sl"][:] = S
    d = {n: to_dev(a) for n, a in c.items()}
    a, la = ops.prefix_attention(d["q"], d["kp"], d["vp"], d["ks"], d["vs"])
    k = torch.cat([d["kp"].repeat_interleave(K, 0), d["ks"]], 1).contiguous()
    v = torch.cat([d["vp"].repeat_interleave(K, 0), d["vs"]], 1).contiguous()
    b, lb = ops.prefix_attention(d["q"], k_suffix=k, v_suffix=v)
    assert (a.float() - b.float()).abs().max() <= 2.0 ** -7 * b.float().abs().max()
    assert (la - lb).abs().max() < 1e-4


def test_attention_bindings_refuse():
    q = torch.zeros((4, 4, 64), device="cuda:0")
    k = torch.zeros((2, 10, 2, 64), device="cuda:0")
    s = torch.zeros((4, 3, 2, 64), device="cuda:0")
    i = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda:0")
    for bad in (dict(q=q[0]), dict(k_prefix=None), dict(v_prefix=k[:1]), dict(k_suffix=s),
                dict(k_suffix=s[:3], v_suffix=s[:3]), dict(prefix_len=i(1)),
                dict(suffix_len=i(1, 2)), dict(group_offsets=i(0, 4)), dict(v_prefix=k.bfloat16()),
                dict(out=q[:1]), dict(k_prefix=None, v_prefix=None),
                dict(k_prefix=k.transpose(0, 1), v_prefix=k.transpose(0, 1)),
                dict(prefix_len=torch.zeros(2, dtype=torch.int32))):
        a = dict(q=q, k_prefix=k, v_prefix=k)
        a.update(bad)
        with pytest.raises(ValueError):
            ops.prefix_attention(**a)
    with pytest.raises(ops.MoeError):
        ops.prefix_attention(q[:3], k, k)             # three rows, two equal groups
    with pytest.raises(ops.MoeError):
        ops.prefix_attention(q[..., :36].contiguous(), k[..., :36].contiguous(),
                             k[..., :36].contiguous())
    with pytest.raises(TypeError):
        ops.prefix_attention(q.half(), k.half(), k.half())
