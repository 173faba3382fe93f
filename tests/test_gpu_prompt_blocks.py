"""Every kind of block of moe_prompt_attention against the float64 oracle: eight waves,
and one, two or four groups of four, with and without splits, of every padded dimension
and type. `_plan` repeats the library's choice with the limits that its source holds, so
that a limit that is moved fails here instead of leaving a kind untested."""
import os
import re

import numpy as np
import pytest
import torch

from paper_2410_17954_amd import ops
from gpu_helpers import to_dev
from test_gpu_prompt_attention import _case, _check

SOURCE = os.path.join(os.path.dirname(ops.__file__), "csrc", "prompt_attention.hip")


def _limits():
    text = open(SOURCE).read()
    return {n: int(v) for n, v in re.findall(r"\b(k\w+) = (\d+)[,;]", text)}


def _plan(N, M, B, Hq, Hkv, D, dtype):
    """(waves, groups, splits, whole columns of a block) as pr_plan chooses them."""
    k = _limits()
    nq, up = Hq // Hkv, lambda a, b: -(-a // b)
    keys = up(M, B)
    wide = dtype == "bf16" and keys >= k["kWideKeys"] and up(N, B) * nq >= k["kWideColumns"]
    dp = 64 if D <= 64 else 128 if D <= 128 else 256
    bm = 16 * (2 if wide and dp < 256 else 1) * (8 if wide else 4)
    most = min(max(1, keys // k["kMinKeys"]), k["kMostSplits"])
    some = min(B, N)
    cols = up(N, some) * nq
    used = some * up(cols, bm) * Hkv
    groups = 1
    if not wide and used <= k["kGroupBlocks"] and keys >= k["kGroupKeys"] and \
            (dtype == "bf16" or dp == 64):
        groups = 2
    if not wide and dtype == "bf16" and dp <= 128 and used <= k["kFourBlocks"] and \
            keys >= k["kFourKeys"] and cols >= k["kFourColumns"]:
        groups = 4
    want = k["kFourBlocks"] if groups == 4 else k["kWideSplitBlocks"] if wide else \
        k["kSplitBlocks"] if dtype == "bf16" else k["kFloatSplitBlocks"]
    fit = max(1, keys // k["kFourMinKeys"]) if groups == 4 else most
    return 8 if wide else 4, groups, min(fit, most, max(1, want // used)), bm


# waves, groups, split or not; type, heads, dimension, queries and keys of each sequence
KINDS = [
    (8, 1, 1, "bf16", 8, 2, 64, [333], [4300]),
    (8, 1, 1, "bf16", 8, 2, 40, [70, 300], [4097, 4200]),
    (8, 1, 0, "bf16", 16, 8, 64, [4200], [4200]),
    (8, 1, 1, "bf16", 8, 2, 128, [301], [4203]),
    (8, 1, 1, "bf16", 7, 1, 80, [90, 257, 1], [4500, 4200, 4001]),
    (8, 1, 0, "bf16", 16, 8, 128, [4200], [4211]),
    (8, 1, 0, "bf16", 40, 8, 80, [1100], [4100]),
    (8, 1, 1, "bf16", 8, 2, 256, [131], [4300]),
    (8, 1, 1, "bf16", 4, 1, 200, [300, 75], [4100, 4350]),
    (8, 1, 0, "bf16", 32, 8, 256, [700], [4150]),
    (4, 1, 0, "bf16", 8, 2, 64, [100, 33], [100, 40]),
    (4, 1, 1, "bf16", 8, 2, 64, [20], [400]),
    (4, 2, 0, "bf16", 32, 8, 64, [600], [600]),
    (4, 2, 1, "bf16", 8, 2, 48, [20, 9], [900, 700]),
    (4, 4, 0, "bf16", 8, 2, 64, [300], [333]),
    (4, 4, 1, "bf16", 8, 2, 32, [260], [1500]),
    (4, 1, 0, "bf16", 8, 2, 128, [100, 33], [100, 40]),
    (4, 1, 1, "bf16", 8, 2, 96, [20], [400]),
    (4, 2, 0, "bf16", 32, 8, 128, [600], [600]),
    (4, 2, 1, "bf16", 8, 2, 128, [20, 9], [900, 700]),
    (4, 4, 0, "bf16", 8, 2, 80, [300], [333]),
    (4, 4, 1, "bf16", 8, 2, 128, [260], [1500]),
    (4, 1, 0, "bf16", 8, 2, 256, [60], [100]),
    (4, 1, 1, "bf16", 8, 2, 192, [100], [300]),
    (4, 2, 0, "bf16", 32, 8, 256, [600], [600]),
    (4, 2, 1, "bf16", 8, 2, 136, [50], [900]),
    (4, 1, 0, "f32", 8, 2, 64, [100], [100]),
    (4, 1, 1, "f32", 8, 2, 40, [50], [400]),
    (4, 2, 0, "f32", 48, 12, 64, [600], [600]),
    (4, 2, 1, "f32", 8, 2, 64, [50, 70], [900, 600]),
    (4, 1, 0, "f32", 8, 2, 128, [100], [110]),
    (4, 1, 1, "f32", 8, 2, 72, [50], [600]),
    (4, 1, 0, "f32", 8, 2, 256, [100], [110]),
    (4, 1, 1, "f32", 8, 2, 200, [50], [600]),
]


@pytest.mark.parametrize("waves,groups,split,dtype,Hq,Hkv,D,nq,nk", KINDS)
def test_kinds_are_what_they_are_listed_as(waves, groups, split, dtype, Hq, Hkv, D, nq, nk):
    w, g, s, _ = _plan(sum(nq), sum(nk), len(nq), Hq, Hkv, D, dtype)
    assert (w, g, int(s > 1)) == (waves, groups, split)
    if split:                                        # what it needs is what the query asks for
        need = ops.prompt_attention_workspace(sum(nq), sum(nk), len(nq), Hq, Hkv, D,
                                              ops.MOE_BF16 if dtype == "bf16" else ops.MOE_F32)
        assert need >= s * sum(nq) * Hq * (4 * D + 8)


def test_every_kind_is_listed():
    listed = {(w, g, split, dtype, 64 if D <= 64 else 128 if D <= 128 else 256)
              for w, g, split, dtype, _, _, D, _, _ in KINDS}
    for split in (0, 1):
        for dp in (64, 128, 256):
            assert {(8, 1, split, "bf16", dp), (4, 1, split, "bf16", dp), (4, 2, split, "bf16", dp),
                    (4, 1, split, "f32", dp)} <= listed
        assert {(4, 4, split, "bf16", 64), (4, 4, split, "bf16", 128), (4, 2, split, "f32", 64)} <= listed


@pytest.mark.gpu
@pytest.mark.parametrize("waves,groups,split,dtype,Hq,Hkv,D,nq,nk", KINDS)
def test_kind(waves, groups, split, dtype, Hq, Hkv, D, nq, nk):
    c, _ = _case(dtype, nq, nk, Hq, Hkv, D, sum(nk) + D + Hq, before=1, after=2)
    bm = _plan(sum(nq), sum(nk), len(nq), Hq, Hkv, D, dtype)[3]
    # first and last tokens, around the ends of blocks' and of waves' columns
    rows, n_q = set(), Hq // Hkv
    for b, n in enumerate(nq):
        at = [0, 1, n - 2, n - 1, n // 2]
        for cols in (16, bm // 2, bm, 2 * bm, n * n_q // bm * bm):
            at += [cols // n_q - 1, cols // n_q]
        rows |= {int(c["qo"][b]) + i for i in at if 0 <= i < n}
    a = _check(c, dtype, D ** -0.5, rows=rows)
    b = _check(c, dtype, D ** -0.5, rows={1})
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])

    # values that are no numbers: of keys that all queries see, and of a query's own
    d = {x: to_dev(c[x]) for x in ("q", "k", "v", "qo", "ko")}
    per, past = Hq // Hkv, nk[0] - nq[0]
    for key, h, dim, x in ((past + nq[0] // 2, Hkv - 1, D - 1, float("nan")),
                           (past // 2, 0, 3, float("-inf"))):
        v = d["v"].clone()
        v[key, h, dim] = x
        out, lse = ops.prompt_attention(d["q"], d["k"], v, q_offsets=d["qo"], k_offsets=d["ko"])
        want = a[0][1:-2].clone()
        want[max(0, key - past):nq[0], h * per:(h + 1) * per, dim] = x
        got = out[1:-2]
        same = (got == want) | (torch.isnan(got) & torch.isnan(want))
        assert same.all(), (key, (~same).nonzero()[:4])
        assert torch.equal(lse[1:-2], a[1][1:-2])
