"""The decode-step operators at the edges of their contracts, beside the tests of
each: scores that swallow the logits, routes without a number."""
import numpy as np
import pytest
import torch

import oracle
from paper_2410_17954_amd import ops, synth
from gpu_helpers import to_dev, to_host, vals
from test_gpu_beam import _bound
from test_gpu_layer_decode import _check, _expert_bound, _f, _inputs

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
LOW = np.finfo(np.float32).min


def _swallowed(dtype, V):
    """Logits that float64 no longer tells apart beside a score of -1e9 (its step
    is 1.2e-7), the same in all four rows, the largest far behind, two equal."""
    g = np.random.default_rng(V)
    z = (1e-9 * g.standard_normal(V)).astype(np.float32)
    z[V - 5], z[[7, V // 2]] = 9e-9, 8e-9
    z = np.broadcast_to(z, (1, 4, V))
    bits = synth.bf16_bits(z) if dtype == "bf16" else np.ascontiguousarray(z)
    return bits, synth.values(bits) if dtype == "bf16" else z.astype(np.float64)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scores", [
    [-1e9] * 4, [-1e30] * 4, [LOW] * 4, [-np.inf, LOW, -np.inf, -1e30], [np.inf, 0, 0, np.inf],
    [-1e9, 0, LOW, -1e30],
])
@pytest.mark.parametrize("n", [4, 20])
def test_scores_that_swallow_the_logits(n, scores, dtype):
    """Dead beams carry -1e9 or the lowest number: within a beam the larger logit
    comes first though the sums are equal, and a request's result does not depend on
    how many others there are (which sets the length of a row's chunks)."""
    V = 32000
    bits, z = _swallowed(dtype, V)
    s = np.array([scores], np.float32)
    rp, rt, rs, _ = oracle.beam_select(z, s, n)
    for B in (1, 64):
        zd = to_dev(bits).repeat(B, 1, 1)
        parent, token, score, _ = ops.beam_select(zd, to_dev(np.repeat(s, B, 0)), n)
        parent = to_host(parent) - 4 * np.arange(B)[:, None]
        assert (parent == rp).all() and (to_host(token) == rt).all()
        score = to_host(score).astype(np.float64)
        finite = np.isfinite(rs[0])
        assert (score[:, ~finite] == rs[0, ~finite]).all()
        assert (np.abs(score[:, finite] - rs[:, finite]) <= _bound(rs[0, finite], V)).all()


def _layer_bound(d, ref, u):
    """The bound of test_gpu_layer_decode on every output of a layer whose slots are
    its experts."""
    x, (wg, wu, wd) = _f(d["x"]), (_f(d[n]) for n in ("w_gate", "w_up", "w_down"))
    n = ref["idx"].shape[1] * wg.shape[1] + (0 if d["shared"] is None else d["shared"][0].shape[0])
    bound = u * np.abs(ref["y"]) + 2.0 ** -23 * np.abs(ref["y"])
    for e in np.unique(ref["idx"]):
        gate = np.where(ref["idx"] == e, ref["w"], 0).sum(1)[:, None]
        bound += _expert_bound(x, wg[e], wu[e], wd[e], gate, u, n)
    if d["shared"] is not None:
        bound += _expert_bound(x, *(_f(t) for t in d["shared"]), 1.0, u, n)
    return bound * (1 + u) + 1e-37


@pytest.mark.parametrize("renorm", [True, False])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,E,Fs", [(5, 7, 0), (16, 40, 24), (40, 130, 24)])
def test_routes_of_masks_that_leave_little(T, E, Fs, dtype, renorm):
    """A NaN logit counts for nothing (as one that a mask pushes down to nothing), a
    token whose mask leaves no expert has none, and neither touches the others."""
    H, F, k = 64, 40, 3
    d, g = _inputs(T, H, F, E, E, dtype, T + E, Fs)
    args = [to_dev(d[n]) for n in ("x", "w_router", "w_gate", "w_up", "w_down")]
    sh = None if d["shared"] is None else tuple(to_dev(t) for t in d["shared"])

    def call(bias):
        return ops.layer_decode(*args, k, bias=to_dev(bias), renormalize=renorm, shared=sh)

    nan = g.standard_normal((T, E)).astype(np.float32)
    nan[1, [0, E - 2]] = np.nan
    nan[T - 2, k:] = np.nan                  # k numbers left
    low = np.where(np.isnan(nan), np.float32(-1e30), nan)
    masked, _ = _check(d, k, dtype, bias=low, renorm=renorm)
    for a, b in zip(call(nan), masked):
        assert torch.equal(a, b)
    empty, rest = [2, T - 1], [t for t in range(T) if t not in (2, T - 1)]
    nan[2] = -np.inf                         # nothing left
    nan[T - 1], nan[T - 1, 4] = -np.inf, np.nan
    y, idx, w, inc = call(nan)
    assert torch.equal(idx[rest], masked[1][rest]) and torch.equal(w[rest], masked[2][rest])
    assert (idx[empty] == -1).all() and (w[empty] == 0).all() and (inc == 0).all()
    f = {n: _f(d[n]) for n in ("x", "w_router", "w_gate", "w_up", "w_down")}
    shared = None if sh is None else tuple(_f(t) for t in d["shared"])
    ref = oracle.moe_layer(f["x"], f["w_router"], k, f["w_gate"], f["w_up"], f["w_down"],
                           bias=low.astype(np.float64), renormalize=renorm, shared=shared)
    ref["w"][empty] = 0
    ref["y"][empty] = 0
    if shared is not None:
        a = f["x"][empty] @ shared[0].T
        ref["y"][empty] = (a / (1 + np.exp(-a)) * (f["x"][empty] @ shared[1].T)) @ shared[2].T
    u = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    assert (np.abs(vals(y) - ref["y"]) <= _layer_bound(d, ref, u)).all()


def test_select_of_a_shrinking_batch_on_one_workspace():
    """One buffer, sized for the first step, while requests end: long chunks, then
    short ones (more lists than the long ones had)."""
    g = torch.Generator(device=DEV).manual_seed(3)
    K, V, n = 8, 128000, 16
    z = torch.randn((16, K, V), device=DEV, generator=g).bfloat16()
    s = torch.randn((16, K), device=DEV, generator=g)
    size = ops.beam_select_workspace(16, K, V, n)
    guard = torch.full((size + 4096,), 0x5a, dtype=torch.uint8, device=DEV)
    ws = guard[2048:2048 + size]
    first = None
    for B in (16, 9, 4, 3, 2, 1):
        parent, token, score, _ = ops.beam_select(z[:B], s[:B], n, workspace=ws)
        if first is None:
            first = parent, token, score
        assert torch.equal(parent, first[0][:B]) and torch.equal(token, first[1][:B])
        assert (score - first[2][:B]).abs().max() < 1e-5
    assert (guard[:2048] == 0x5a).all() and (guard[2048 + size:] == 0x5a).all()


@pytest.mark.parametrize("P", [700, 16384])
def test_attention_of_a_shrinking_batch_on_one_workspace(P):
    """One buffer, sized for the first step, while sequences end: other column tiles,
    other splits, more of the buffer for fewer rows."""
    g = torch.Generator(device=DEV).manual_seed(3)
    R, Hq, Hkv, D, S = 49, 32, 8, 128, 500
    q, ks, vs, kp, vp = (torch.randn(s, device=DEV, generator=g).bfloat16() for s in (
        (R, Hq, D), (R, S, Hkv, D), (R, S, Hkv, D), (1, P, Hkv, D), (1, P, Hkv, D)))
    size = ops.prefix_attention_workspace(R, 1, Hq, Hkv, D, P, S)
    guard = torch.full((size + 4096,), 0x5a, dtype=torch.uint8, device=DEV)
    ws = guard[2048:2048 + size]
    for n in (49, 48, 33, 32, 31, 17, 16, 15, 5, 4, 2, 1):
        out, lse = ops.prefix_attention(q[:n], kp, vp, ks[:n], vs[:n], workspace=ws)
        own, own_lse = ops.prefix_attention(q[:n], kp, vp, ks[:n], vs[:n])
        assert torch.equal(out, own) and torch.equal(lse, own_lse)
    assert (guard[:2048] == 0x5a).all() and (guard[2048 + size:] == 0x5a).all()


def test_reorder_of_caches_that_touch():
    """Keys and values in one allocation, one right behind the other: apart. One that
    begins inside the other: refused, nothing moved."""
    both = torch.arange(2 * 2 * 4 * 3 * 16, device=DEV, dtype=torch.int32).view(2, 2, 4, 3, 16)
    keep = both.clone()
    parent = torch.tensor([[1, 0], [3, 3]], dtype=torch.int32, device=DEV)
    flat = both.view(-1)
    n = both[0].numel()
    with pytest.raises(ops.MoeError):
        ops.beam_reorder([flat[:n].view(2, 4, 3, 16), flat[n - 4:2 * n - 4].view(2, 4, 3, 16)], parent)
    assert torch.equal(both, keep)
    ops.beam_reorder([both[1], both[0]], parent)
    assert torch.equal(both, keep[:, :, [1, 0, 3, 3]])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,P,S", [(2, 30, 5), (3, 900, 40), (70, 300, 3), (40, 0, 20)])
def test_rows_whose_scores_are_all_minus_infinity(rows, P, S, dtype):
    """As rows without a key, beside rows whose suffix has one key left."""
    g = torch.Generator(device=DEV).manual_seed(P)
    Hq, Hkv, D = 8, 2, 64
    q, ks, vs, kp, vp = (torch.randn(s, device=DEV, generator=g).to(dtype) for s in (
        (rows, Hq, D), (rows, S, Hkv, D), (rows, S, Hkv, D), (1, P, Hkv, D), (1, P, Hkv, D)))
    q[..., 0] = 1.0
    kp[..., 0], ks[..., 0] = -float("inf"), -float("inf")
    ks[1::2, S - 1, :, 0] = 0.0
    prefix = (kp, vp) if P else (None, None)
    out, lse = ops.prefix_attention(q, *prefix, ks, vs)
    assert (out[::2] == 0).all() and (lse[::2] == -float("inf")).all()
    # The only key that counts: its value. The exponential is that of the rounding of its
    # own score, p = 2^r, |r| below 2^-24 of a score of at most 64 (log2), so p need not
    # be one. float32: (p v) (1 / p) with a product of the matrix cores (2^-23, either
    # way), a division and a product (2^-24 each), 2^-22 together. bf16: p is 1 as an
    # operand, and 1 / p is within 2^-17 of 1, which a value of eight bits rounds to itself.
    want = vs[1::2, S - 1].repeat_interleave(Hq // Hkv, 1)
    tol = 0.0 if dtype == torch.bfloat16 else 2.0 ** -22
    assert ((out[1::2].double() - want.double()).abs() <= tol * want.double().abs()).all()
    s = (q[1::2].double() * ks[1::2, S - 1].double().repeat_interleave(Hq // Hkv, 1)).sum(-1) / 8
    # a float32 sum of 64 products of at most 20 each, times log2 e and back
    assert (lse[1::2] - s).abs().max() <= 2 * 65 * 2.0 ** -24 * 64 * 20 / 8
