"""CPU checks of the decode step's workspace sizes: what the largest call of a loop
needs serves the smaller ones, as when sequences end and the batch shrinks."""
import itertools
import os

import pytest

from paper_2410_17954_amd import ops
from paper_2410_17954_amd.build import library_path


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(library_path()):
        from paper_2410_17954_amd import build
        build.build(verbose=False)
    return ops.load_library()


def _never_falls(size, *axes):
    """size(point) over the grid of the axes (each ascending): no neighbour with one
    coordinate larger is smaller."""
    grid = {p: size(*(a[i] for a, i in zip(axes, p)))
            for p in itertools.product(*(range(len(a)) for a in axes))}
    for p, n in grid.items():
        assert n > 0, p
        for d in range(len(p)):
            q = p[:d] + (p[d] + 1,) + p[d + 1:]
            if q in grid:
                assert n <= grid[q], [(a[i], a[j]) for a, i, j in zip(axes, p, q)]


def test_select_workspace_of_the_largest_call_serves_all():
    _never_falls(ops.beam_select_workspace, list(range(1, 70)) + [127, 128, 129, 255, 256, 1000],
                 [1, 2, 3, 4, 5, 8, 9, 31, 32],
                 [1, 2047, 2048, 2049, 16384, 16385, 32000, 32769, 128000, 128256, 151936],
                 [1, 4, 16, 64])


@pytest.mark.parametrize("dtype", [ops.MOE_BF16, ops.MOE_F32])
@pytest.mark.parametrize("Hq,Hkv,D", [(32, 8, 128), (16, 16, 64), (8, 1, 80), (64, 2, 256), (3, 3, 40)])
def test_attention_workspace_of_the_largest_call_serves_all(Hq, Hkv, D, dtype):
    keys = [0, 1, 127, 128, 129, 500, 4096, 65536]
    rows = list(range(1, 70)) + [127, 128, 129, 500, 1000]
    for G in (1, 2, 5, 16, 64):
        _never_falls(lambda r, p, s: 1 + ops.prefix_attention_workspace(r, G, Hq, Hkv, D, p, s, dtype),
                     [r for r in rows if r >= G], keys, keys[::2])
    for R in (64, 70, 1000):
        _never_falls(lambda g, p: ops.prefix_attention_workspace(R, g, Hq, Hkv, D, p, 30, dtype),
                     list(range(1, 65)), keys)


@pytest.mark.parametrize("H,F,Fs", [(2048, 1408, 5632), (4096, 14336, 0), (72, 56, 24)])
def test_layer_workspace_of_the_most_tokens_serves_all(H, F, Fs):
    for dtype in (ops.MOE_BF16, ops.MOE_F32):
        _never_falls(lambda t: ops.layer_decode_workspace(t, H, F, 60, 4, Fs, dtype), list(range(1, 65)))
