"""The decode-step operators at the edges of their contracts, beside the tests of
each: scores that swallow the logits, routes without a number."""
import numpy as np
import pytest
import torch

import oracle
from paper_2410_17954_amd import ops, synth
from gpu_helpers import to_dev, to_host
from test_gpu_beam import _bound

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
