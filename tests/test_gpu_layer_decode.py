"""moe_layer_decode against the float64 oracle's layer: experts and flags bit for
bit, gates and outputs within bounds from the roundings.

Gates: float32 exponentials of float64 differences and their sums, 2^-20
relative. Outputs: with u the type's half step (2^-8 bf16, 2^-24 float32),
  a' = w silu(g) u'   g, u' float32 sums of H products, one rounding of a',
  y  = sum of a' . w_down (float32 sum of n = rows of all experts), one rounding.
g and u' are off by at most G = 2 (H + 1) 2^-24 S_g, S_g the sum of the absolute
products (the factor 2: matrix-core additions may round either way); silu has a
slope of at most 1.1. So |dy| <= 2^-8 |y| + sum |w_down| (|a'| (u + 2^-20 +
n 2^-23) + w (1.1 G_g |u'| + |silu(g)| G_u)), evaluated in float64 per output."""
import numpy as np
import pytest
import torch

import oracle
from paper_2410_17954_amd import ops, synth
from gpu_helpers import to_dev, to_host, vals

pytestmark = pytest.mark.gpu


def _inputs(T, H, F, E, S, dtype, seed, Fs=0, scale=0.1):
    g = np.random.default_rng(seed)

    def draw(*shape, std=scale):
        a = (std * g.standard_normal(shape)).astype(np.float32)
        return synth.bf16_bits(a) if dtype == "bf16" else a

    d = dict(x=draw(T, H, std=1.0), w_router=draw(E, H), w_gate=draw(S, F, H), w_up=draw(S, F, H),
             w_down=draw(S, H, F), shared=None)
    if Fs:
        d["shared"] = (draw(Fs, H), draw(Fs, H), draw(H, Fs))
    return d, g


def _f(a):
    return synth.values(a) if a.dtype == np.uint16 else a.astype(np.float64)


def _expert_bound(x, wg, wu, wd, gate, u, n):
    """The bound on |dy| that one expert's rows add, gates [rows, 1]."""
    H = x.shape[1]
    gam = 2 * (H + 1) * 2.0 ** -24
    g, up = x @ wg.T, x @ wu.T
    Gg, Gu = gam * (np.abs(x) @ np.abs(wg).T), gam * (np.abs(x) @ np.abs(wu).T)
    silu = g / (1 + np.exp(-g))
    a = gate * np.abs(silu * up)
    rel = u + 2.0 ** -20 + n * 2.0 ** -23
    # 4 2^-24: silu's own rounding, hardware exponential and reciprocal included in 2^-20
    da = a * rel + gate * (1.1 * Gg * np.abs(up) + np.abs(silu) * Gu + 1.1 * Gg * Gu)
    return da @ np.abs(wd).T


def _check(d, k, dtype, bias=None, renorm=True, slot=None, accumulate=None, out=None, **kw):
    args = {n: to_dev(d[n]) for n in ("x", "w_router", "w_gate", "w_up", "w_down")}
    sh = None if d["shared"] is None else tuple(to_dev(t) for t in d["shared"])
    y = None if accumulate is None else to_dev(accumulate)
    got = ops.layer_decode(*args.values(), k, bias=None if bias is None else to_dev(bias),
                           renormalize=renorm, slot_of_expert=None if slot is None else to_dev(slot),
                           shared=sh, y=y, accumulate=accumulate is not None, **kw)
    torch.cuda.synchronize()
    x = _f(d["x"])
    E = d["w_router"].shape[0]
    sl = np.arange(E) if slot is None else slot
    S = d["w_gate"].shape[0]
    ok_slot = np.where((sl >= 0) & (sl < S), sl, -1)
    shv = None if sh is None else tuple(_f(t) for t in d["shared"])
    wg, wu, wd = (_f(d[n]) for n in ("w_gate", "w_up", "w_down"))
    ref = oracle.moe_layer(x, _f(d["w_router"]), k, wg, wu, wd,
                           bias=None if bias is None else bias.astype(np.float64),
                           renormalize=renorm, slot_of_expert=ok_slot, shared=shv)
    yo, idx, w, inc = got
    assert np.array_equal(to_host(idx), ref["idx"])
    assert np.array_equal(to_host(inc), ref["incomplete"])
    wr = ref["w"]
    assert (np.abs(to_host(w) - wr) <= 2.0 ** -20 * wr + 1e-37).all()
    u = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    T, H = x.shape
    F = wg.shape[1]
    n = k * F + (0 if shv is None else shv[0].shape[0])
    bound = np.zeros((T, H))
    for e in np.unique(ref["idx"]):
        s = ok_slot[e]
        if s < 0:
            continue
        gate = np.where(ref["idx"] == e, wr, 0).sum(1)
        t = np.nonzero(gate)[0]
        bound[t] += _expert_bound(x[t], wg[s], wu[s], wd[s], gate[t, None], u, n)
    if shv is not None:
        bound += _expert_bound(x, *shv, 1.0, u, n)
    yr = ref["y"] + (0 if accumulate is None else _f(accumulate))
    bound += u * np.abs(yr) + 2.0 ** -23 * np.abs(yr)
    bound = bound * (1 + u) + 1e-37
    err = np.abs(vals(yo) - yr)
    assert (err <= bound).all(), (err / bound).max()
    return got, (err / bound).max()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,H,F,E,k,Fs", [
    (1, 64, 64, 1, 1, 0), (1, 8, 8, 2, 2, 8), (2, 136, 72, 8, 2, 0), (5, 256, 200, 60, 4, 104),
    (16, 512, 128, 16, 3, 0), (17, 200, 264, 8, 2, 40), (32, 128, 96, 4, 4, 0),
    (33, 320, 80, 33, 5, 88), (48, 96, 136, 7, 1, 0), (64, 264, 120, 64, 6, 64),
    (64, 64, 40, 256, 32, 0), (64, 72, 56, 1, 1, 24),
])
def test_layer_sizes(T, H, F, E, k, Fs, dtype):
    d, g = _inputs(T, H, F, E, E, dtype, T * 1000 + H, Fs)
    _check(d, k, dtype)
    _check(d, k, dtype, bias=g.standard_normal(E).astype(np.float32), renorm=False)


def test_layer_float32_quarters():
    # multiples of four that bfloat16 does not take
    d, g = _inputs(7, 132, 68, 6, 6, "f32", 3, 36)
    _check(d, 2, "f32", bias=g.standard_normal((7, 6)).astype(np.float32))


@pytest.mark.parametrize("T", [1, 9, 40])
def test_layer_misses_and_odd_slots(T):
    E, k = 12, 3
    d, g = _inputs(T, 128, 96, E, 5, "bf16", T, 0)
    slot = np.full(E, -1, np.int32)
    slot[[1, 4, 7, 8, 11]] = [3, 0, 4, 2, 1]
    _check(d, k, "bf16", slot=slot)
    slot[0], slot[5] = 5, -9                 # outside the slots: not resident either
    _check(d, k, "bf16", slot=slot)
    _check(d, k, "bf16", slot=np.full(E, -1, np.int32))        # nothing resident: zeros
    # nothing resident and a y to add to: unchanged
    y0 = synth.bf16_bits(g.standard_normal((T, 128)).astype(np.float32))
    got, _ = _check(d, k, "bf16", slot=np.full(E, -1, np.int32), accumulate=y0)
    assert np.array_equal(to_host(got[0]), y0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_layer_accumulate_and_in_place(dtype):
    T, H = 11, 256
    d, g = _inputs(T, H, 160, 8, 8, dtype, 5, 72)
    y0 = g.standard_normal((T, H)).astype(np.float32)
    y0 = synth.bf16_bits(y0) if dtype == "bf16" else y0
    _check(d, 2, dtype, accumulate=y0)
    # y = x: the layer of x, over it
    args = [to_dev(d[n]) for n in ("x", "w_router", "w_gate", "w_up", "w_down")]
    sh = tuple(to_dev(t) for t in d["shared"])
    apart = ops.layer_decode(*args, 2, shared=sh)[0]
    same = ops.layer_decode(*args, 2, shared=sh, y=args[0])[0]
    assert same is args[0] and torch.equal(apart, same)


def test_layer_ties_and_near_ties():
    # equal router rows tie exactly; a last-bit difference decides
    T, H, E, k = 20, 512, 24, 5
    d, g = _inputs(T, H, 32, E, E, "bf16", 8)
    wr = d["w_router"]
    wr[5], wr[17], wr[11] = wr[2], wr[2], wr[3]
    wr[20] = wr[9]
    wr[20, 77] ^= 1
    _check(d, k, "bf16")
    _check(d, k, "bf16", bias=np.repeat(np.float32([0.5, 0.25]), E // 2))


def test_layer_many_rows_on_one_expert_and_repeats():
    # a bias sends all tokens to the same two experts; repeated calls on a
    # workspace full of other values give the same bits
    T, H, F, E = 64, 256, 136, 16
    d, _ = _inputs(T, H, F, E, E, "bf16", 12, 64)
    bias = np.zeros(E, np.float32)
    bias[[3, 14]] = 50
    got, _ = _check(d, 2, "bf16", bias=bias)
    ws = ops.workspace_tensor(ops.layer_decode_workspace(T, H, F, E, 2, 64), "cuda:0")
    args = [to_dev(d[n]) for n in ("x", "w_router", "w_gate", "w_up", "w_down")]
    sh = tuple(to_dev(t) for t in d["shared"])
    for fill in (0, 255, 127):
        ws.fill_(fill)
        again = ops.layer_decode(*args, 2, bias=to_dev(bias), shared=sh, workspace=ws)
        for a, b in zip(got, again):
            assert torch.equal(a, b)


def test_layer_nan_logits():
    # float32: a NaN logit is never chosen; too few numbers leave -1 and gate 0
    T, H, E = 2, 32, 4
    d, _ = _inputs(T, H, 32, E, E, "f32", 2)
    bias = np.zeros((T, E), np.float32)
    bias[0, 1] = np.nan
    bias[1, :3] = np.nan
    args = [to_dev(d[n]) for n in ("x", "w_router", "w_gate", "w_up", "w_down")]
    _, idx, w, inc = ops.layer_decode(*args, 3, bias=to_dev(bias))
    idx, w = to_host(idx), to_host(w)
    assert sorted(idx[0].tolist()) == [0, 2, 3] and idx[1].tolist() == [3, -1, -1]
    assert w[1].tolist() == [1.0, 0.0, 0.0]
    assert to_host(inc).tolist() == [0, 0]


@pytest.mark.parametrize("name,T", [("qwen15_moe_layer", 3), ("qwen15_moe_layer", 50),
                                    ("deepseek_v2_lite_layer", 8)])
def test_layer_against_the_four_calls(name, T):
    """Workload shapes: the same experts, gates within a step, outputs within the
    bf16 bound of the chain's own test."""
    c = synth.workload(name)
    H, F, E, k, ns = c["H"], c["F"], c["E"], c["k"], c["n_shared"]
    g = torch.Generator(device="cuda:0").manual_seed(T)
    bf = lambda *s: torch.empty(s, dtype=torch.bfloat16, device="cuda:0").normal_(0, 0.02, generator=g)
    x = bf(T, H) * 50
    wr, wg, wu, wd = bf(E, H), bf(E, F, H), bf(E, F, H), bf(E, H, F)
    sh = (bf(ns * F, H), bf(ns * F, H), bf(H, ns * F))
    idx, w, _ = ops.route(x, wr, k, renormalize=False)
    off, rop, _, xp = ops.permute(x, idx, E)
    yp = ops.expert_ffn(xp, off, wg, wu, wd)
    so = torch.tensor([0, T], dtype=torch.int32, device="cuda:0")
    ys = ops.expert_ffn(x, so, sh[0][None], sh[1][None], sh[2][None])
    y, _ = ops.combine(yp, idx, w, rop, y_shared=ys)
    y2, idx2, w2, _ = ops.layer_decode(x, wr, wg, wu, wd, k, renormalize=False, shared=sh)
    assert torch.equal(idx, idx2)
    assert torch.allclose(w, w2, rtol=2e-6, atol=0)
    assert (y.float() - y2.float()).abs().max() <= 1e-2 * y.float().abs().max()


def test_layer_bindings_refuse():
    d, _ = _inputs(2, 64, 32, 4, 4, "bf16", 1)
    x, wr, wg, wu, wd = (to_dev(d[n]) for n in ("x", "w_router", "w_gate", "w_up", "w_down"))
    for bad in (dict(w_up=wu[:, :16].contiguous()), dict(w_down=wu), dict(x=x[0]),
                dict(w_router=wr.float()), dict(y=x[:1]), dict(accumulate=True),
                dict(bias=wr), dict(shared=(wg[0], wu[0], wu[0])), dict(x=x.cpu()),
                dict(slot_of_expert=torch.zeros(3, dtype=torch.int32, device="cuda:0"))):
        a = dict(x=x, w_router=wr, w_gate=wg, w_up=wu, w_down=wd, k=2)
        a.update(bad)
        with pytest.raises(ValueError):
            ops.layer_decode(**a)
    with pytest.raises(ops.MoeError):
        ops.layer_decode(x.repeat(40, 1), wr, wg, wu, wd, 2)
    with pytest.raises(ops.MoeError):
        ops.layer_decode(x, wr, wg, wu, wd, 5)
