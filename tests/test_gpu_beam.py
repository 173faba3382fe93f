"""moe_beam_select and moe_beam_reorder against the float64 oracle: parents,
tokens, flags and moved bytes bit for bit. Scores: the result is rounded to
float32 once (2^-24 of it). Its log-sum-exp comes from float32 exponentials: a
term of weight p = exp(-d) / sum carries d 2^-23 (the product with log2 e and its
rounding; d itself is exact or half a step off), 2^-22 of the hardware
exponential, and at most 31 additions of half a step; summed with the weights p
that is at most (mean d + 18) 2^-23, and the mean of d under a row's softmax is
at most ln V (d = ln(1 / p) - ln(1 / p_max), and the entropy is at most ln V)."""
import numpy as np
import pytest
import torch

import oracle
from paper_2410_17954_amd import ops, synth
from gpu_helpers import to_dev, to_host

pytestmark = pytest.mark.gpu


def _logits(g, B, K, V, dtype, kind="normal"):
    if kind == "ties":                              # few distinct values
        z = g.integers(0, 3, size=(B, K, V)).astype(np.float32)
    elif kind == "equal":
        z = np.full((B, K, V), 1.5, np.float32)
    elif kind == "rising":                          # the best tokens all in one place
        z = np.broadcast_to(np.linspace(-4, 9, V, dtype=np.float32), (B, K, V)).copy()
    else:
        z = (2.5 * g.standard_normal((B, K, V))).astype(np.float32)
        z[..., g.integers(0, V, size=3)] += 8.0
    if dtype == "bf16":
        bits = synth.bf16_bits(z)
        return bits, synth.values(bits)
    return z, z.astype(np.float64)


def _bound(score, V):
    return 2.0 ** -24 * np.abs(score) + (np.log(V) + 18) * 2.0 ** -23


def _check_select(zd, z, s, n, finished=None, eos=None):
    fin = None if finished is None else to_dev(finished)
    parent, token, score, done = ops.beam_select(zd, to_dev(s), n, finished=fin, eos=eos)
    rp, rt, rs, rd = oracle.beam_select(z, s, n, finished, eos)
    assert np.array_equal(to_host(parent), rp)
    assert np.array_equal(to_host(token), rt)
    got = to_host(score).astype(np.float64)
    none = rp < 0
    assert np.array_equal(got == -np.inf, none)
    assert (np.abs(got[~none] - rs[~none]) <= _bound(rs[~none], z.shape[-1])).all()
    if eos is None:
        assert done is None
    else:
        assert np.array_equal(to_host(done), rd)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,K,V,n", [
    (1, 1, 1, 1), (1, 1, 7, 3), (2, 3, 5, 20), (1, 4, 2047, 8), (3, 2, 2049, 4), (2, 5, 8193, 10),
    (1, 4, 32000, 4), (5, 8, 16385, 16), (1, 32, 1000, 64), (70, 4, 9001, 8),
])
def test_select_sizes(B, K, V, n, dtype):
    g = np.random.default_rng(V + n)
    bits, z = _logits(g, B, K, V, dtype)
    s = (-5 * g.random((B, K))).astype(np.float32)
    _check_select(to_dev(bits), z, s, n)


@pytest.mark.parametrize("kind", ["ties", "equal", "rising"])
@pytest.mark.parametrize("V,n", [(3, 8), (700, 64), (5001, 5), (20000, 64)])
def test_select_ties(kind, V, n):
    g = np.random.default_rng(V)
    bits, z = _logits(g, 2, 3, V, "bf16", kind)
    # equal rows and equal scores: beams tie too
    s = np.array([[-1, -1, -1], [-3, -2.3, -3]], np.float32)
    z[:, 1], bits[:, 1] = z[:, 0], bits[:, 0]
    z[:, 2], bits[:, 2] = z[:, 0], bits[:, 0]
    _check_select(to_dev(bits), z, s, n)


def test_select_finished_and_empty_rows():
    g = np.random.default_rng(9)
    B, K, V, eos = 6, 4, 3001, 17
    z = (2 * g.standard_normal((B, K, V))).astype(np.float32)
    s = (-3 * g.random((B, K))).astype(np.float32)
    fin = np.zeros((B, K), np.int32)
    s[0, 1:] = -np.inf                        # the first step: one live beam
    fin[1, :] = 1                             # all finished: K candidates, n of 8
    z[1] = np.nan                             # and what their rows hold does not matter
    fin[2, [0, 3]] = [1, -5]
    z[3, 0, 5] = np.nan                       # a row that is no distribution
    z[3, 1, 6] = np.inf
    z[3, 2, :] = -np.inf                      # a row that allows nothing
    z[4, :, 10:] = -np.inf                    # most tokens masked
    z[4, 0, 9:] = np.finfo(np.float32).min    # masked by the lowest number
    s[5] = [np.nan, -np.inf, 2.0, 0.5]
    _check_select(to_dev(z), z.astype(np.float64), s, 8, fin, eos)
    _check_select(to_dev(z), z.astype(np.float64), s, 64, fin, eos)


def test_select_far_below_zero_and_masked_chunks():
    # whole chunks of -inf beside logits near -1000: shares of chunks add up at
    # the row's own maximum
    V = 30000
    z = np.full((1, 2, V), -np.inf, np.float32)
    z[0, 0, 20000:20050] = -1000 + np.arange(50, dtype=np.float32) / 8
    z[0, 1, 5] = -3.0e38
    s = np.zeros((1, 2), np.float32)
    _check_select(to_dev(z), z.astype(np.float64), s, 6)


def test_select_unaligned_rows_and_reused_buffers():
    g = np.random.default_rng(4)
    B, K, V, n = 3, 3, 4099, 6
    for dtype in ("bf16", "f32"):
        bits, z = _logits(g, B, K, V, dtype)
        flat = to_dev(np.concatenate([bits.ravel()[:1], bits.ravel()]))
        zd = flat[1:].view(B, K, V)           # one element off any wider alignment
        assert zd.data_ptr() % 4 in (0, 2)
        s = (-5 * g.random((B, K))).astype(np.float32)
        _check_select(zd, z, s, n)
    ws = ops.workspace_tensor(ops.beam_select_workspace(B, K, V, n), "cuda:0")
    ws.fill_(255)
    outs = [torch.full((B, n), -9, dtype=torch.int32, device="cuda:0") for _ in range(3)]
    best = torch.empty((B, n), device="cuda:0")
    got = ops.beam_select(zd, to_dev(s), n, eos=1, parent=outs[0], token=outs[1], out_scores=best,
                          out_finished=outs[2], workspace=ws)
    assert got[0] is outs[0] and got[3] is outs[2]
    rp, rt, _, rd = oracle.beam_select(z, s, n, None, 1)
    assert np.array_equal(to_host(outs[0]), rp) and np.array_equal(to_host(outs[1]), rt)
    assert np.array_equal(to_host(outs[2]), rd)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 16, 17, 64])
def test_select_masked_to_few_and_equal_chunks(n, dtype):
    # constrained decoding: all but a few tokens at the lowest number; whole
    # chunks of one value, and chunks sorted either way
    V = 20000
    low = np.finfo(np.float32).min if dtype == "f32" else -3.3895313892515355e38
    z = np.full((1, 4, V), low, np.float32)
    z[0, 0, [3, 9000, 19999]] = [1.0, 2.0, 1.5]
    z[0, 1] = 0.25
    z[0, 2] = np.linspace(-2, 2, V)
    z[0, 3] = np.linspace(2, -2, V)
    bits = synth.bf16_bits(z) if dtype == "bf16" else z
    s = np.array([[0.0, 3.5, 2.1, 1.3]], np.float32)
    _check_select(to_dev(bits), synth.values(bits) if dtype == "bf16" else z.astype(np.float64), s, n)


def test_select_many_requests():
    # more rows than one launch's second dimension takes
    g = np.random.default_rng(5)
    B, K, V, n = 9000, 4, 33, 4
    bits, z = _logits(g, B, K, V, "bf16")
    s = (-5 * g.random((B, K))).astype(np.float32)
    parent, token, _, _ = ops.beam_select(to_dev(bits), to_dev(s), n)
    pick = np.r_[0:40, B - 40:B]
    rp, rt, _, _ = oracle.beam_select(z[pick], s[pick], n)
    # ties across beams are decided by the float64 sums; none lies within 1e-6 here
    assert np.array_equal(to_host(parent)[pick] - (pick * K)[:, None],
                          rp - (np.arange(len(pick)) * K)[:, None])
    assert np.array_equal(to_host(token)[pick], rt)


@pytest.mark.parametrize("unit", [(16,), (4, 24), (1000,), (20,), (7,), (1,)])
@pytest.mark.parametrize("L,B,K,S", [(1, 1, 1, 1), (2, 3, 4, 5), (3, 2, 8, 33), (2, 5, 3, 0),
                                     (1, 2, 32, 40)])
def test_reorder_bytes(L, B, K, S, unit):
    g = np.random.default_rng(L + K + S)
    R = B * K
    caches = [g.integers(0, 256, size=(L, R, S) + unit, dtype=np.uint8) for _ in range(2)]
    # permutations, duplicates, rows that stay
    parent = np.stack([b * K + (g.permutation(K) if b % 2 else g.integers(0, K, size=K))
                       for b in range(B)]).astype(np.int32)
    lens = g.integers(-2, S + 3, size=R).astype(np.int32)
    for use in (None, lens):
        dev = [to_dev(c) for c in caches]
        new, err = ops.beam_reorder(dev, to_dev(parent),
                                    lens=None if use is None else to_dev(use))
        assert int(err) == 0
        for c, d in zip(caches, dev):
            ref, ref_lens, _ = oracle.beam_reorder(c, parent.ravel(), K, use)
            assert np.array_equal(to_host(d), ref)
            assert np.array_equal(to_host(new), ref_lens)


def test_reorder_bad_parents_and_unaligned_caches():
    g = np.random.default_rng(2)
    L, B, K, S = 2, 3, 3, 6
    cache = g.integers(0, 256, size=(L, B * K, S, 32), dtype=np.uint8)
    parent = np.array([[1, -1, 0], [0, 4, 99], [-7, 8, 7]], np.int32)
    flat = torch.zeros(cache.size + 5, dtype=torch.uint8, device="cuda:0")
    dev = flat[5:].view(cache.shape)
    dev.copy_(to_dev(cache))
    new, err = ops.beam_reorder([dev], to_dev(parent))
    ref, ref_lens, bad = oracle.beam_reorder(cache, parent.ravel(), K)
    assert bad and int(err) == 1
    assert np.array_equal(to_host(dev), ref) and np.array_equal(to_host(new), ref_lens)
    assert to_host(flat[:5]).sum() == 0


def test_reorder_offsets_past_32_bits():
    # the last rows of a cache of 5 GiB: row offsets need 64 bits
    L, B, K, S, unit = 5, 1, 4, 16384, 16384
    cache = torch.zeros((L, B * K, S, unit), dtype=torch.uint8, device="cuda:0")
    cache[:, 3, ::1000] = torch.arange(L, dtype=torch.uint8, device="cuda:0")[:, None, None] + 7
    parent = torch.tensor([[3, 1, 2, 3]], dtype=torch.int32, device="cuda:0")
    ops.beam_reorder([cache], parent)
    assert torch.equal(cache[:, 0], cache[:, 3])
    assert int(cache[:, 1:3].max()) == 0 and int(cache[4, 0, 1000, 5]) == 11


def test_bindings_refuse():
    z = torch.zeros((2, 2, 9), device="cuda:0")
    s = torch.zeros((2, 2), device="cuda:0")
    with pytest.raises(ValueError):
        ops.beam_select(z.view(4, 9), s)
    with pytest.raises(ValueError):
        ops.beam_select(z, s.view(4))
    with pytest.raises(TypeError):
        ops.beam_select(z.half(), s)
    with pytest.raises(ValueError):
        ops.beam_select(z, s, finished=torch.zeros((2, 2), dtype=torch.int32, device="cuda:0"))
    with pytest.raises(ValueError):
        ops.beam_select(z.transpose(0, 1), s)               # not contiguous
    with pytest.raises(ValueError):
        ops.beam_select(z, s.cpu())
    with pytest.raises(ops.MoeError):
        ops.beam_select(z, s, n_out=65)
    c = torch.zeros((1, 4, 3, 8), device="cuda:0")
    p = torch.zeros((2, 2), dtype=torch.int32, device="cuda:0")
    with pytest.raises(ValueError):
        ops.beam_reorder([], p)
    with pytest.raises(ValueError):
        ops.beam_reorder([c, c[..., :4].contiguous()], p)
    with pytest.raises(ValueError):
        ops.beam_reorder([c], p.view(4))
    with pytest.raises(ops.MoeError):
        ops.beam_reorder([c, c], p)
