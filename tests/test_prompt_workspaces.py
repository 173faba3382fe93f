"""Workspaces of the entry points of include/moeflow_prompt.h: those that a call needs
are asked for, checked and kept apart from its arrays; moe_token_logprobs needs none."""
import ctypes

import pytest
import torch

from paper_2410_17954_amd import ops
from test_prompt_host import _attend, _logprobs, _prompt, at, lib  # noqa: F401


def test_split_calls_need_a_workspace(lib):          # noqa: F811
    few = dict(N=64, M=30000)
    need = lib.moe_prompt_attention_workspace(64, 30000, 1, 8, 2, 64, 1)
    # a float32 result, a maximum and a sum of at least two splits
    assert need >= 2 * 64 * 8 * (64 * 4 + 8)
    for bad in (dict(ws=None), dict(nbytes=0), dict(nbytes=need - 1),
                dict(ws=ctypes.c_void_p((8 << 44) + 16))):
        assert _prompt(lib, **few, **bad) == ops.MOE_ERR_WORKSPACE, bad
    for bad in (dict(ws=at(5)), dict(ws=at(0)), dict(ws=at(6)), dict(ws=at(3))):
        assert _prompt(lib, **few, **bad) == ops.MOE_ERR_ARG, bad
    need = lib.moe_kv4_attention_workspace(4, 1000, 8, 2, 64)
    assert need >= 2 * 4 * 8 * (64 * 4 + 8)
    for bad in (dict(ws=None), dict(nbytes=0), dict(nbytes=need - 1),
                dict(ws=ctypes.c_void_p((10 << 44) + 16))):
        assert _attend(lib, **bad) == ops.MOE_ERR_WORKSPACE, bad
    for bad in (dict(ws=at(7)), dict(ws=at(8)), dict(ws=at(1)), dict(ws=at(6))):
        assert _attend(lib, **bad) == ops.MOE_ERR_ARG, bad


def test_calls_without_splits_need_none(lib):        # noqa: F811
    assert lib.moe_prompt_attention_workspace(64, 128, 1, 8, 2, 64, 1) == 0
    assert lib.moe_kv4_attention_workspace(4, 128, 8, 2, 64) == 0


@pytest.mark.parametrize("R,V,m,n", [(1, 1, 1, 0), (3, 1000, 2, 4), (300, 152000, 0, 64),
                                     ((1 << 22) - 1, 1 << 24, 1, 1)])
def test_logprobs_need_none(lib, R, V, m, n):        # noqa: F811
    assert lib.moe_token_logprobs_workspace(R, V, m, n) == 0
    # a bad argument is refused as one, with and without a workspace
    for ws in (None, at(6)):
        assert _logprobs(lib, n=65, ws=ws, nbytes=0) == ops.MOE_ERR_UNSUPPORTED


@pytest.mark.gpu
def test_logprobs_use_none():
    lib = ops.load_library()
    z = torch.randn(3, 5000, device="cuda:0")
    tok = torch.tensor([[1], [4999], [7]], dtype=torch.int32, device="cuda:0")
    outs = []
    for ws, nbytes in ((None, 0), (torch.full((64,), 7, dtype=torch.uint8, device="cuda:0"), 3)):
        lp, en = torch.zeros(3, 1, device="cuda:0"), torch.zeros(3, device="cuda:0")
        tt = torch.zeros(3, 4, dtype=torch.int32, device="cuda:0")
        tl = torch.zeros(3, 4, device="cuda:0")
        st = lib.moe_token_logprobs(z.data_ptr(), ops.MOE_F32, 3, 5000, 5000, tok.data_ptr(), 1, 4,
                                    lp.data_ptr(), en.data_ptr(), tt.data_ptr(), tl.data_ptr(),
                                    None if ws is None else ws.data_ptr(), nbytes,
                                    torch.cuda.current_stream().cuda_stream)
        assert st == ops.MOE_OK
        outs.append((lp, en, tt, tl))
        assert ws is None or (ws == 7).all()
    assert all(torch.equal(a, b) for a, b in zip(*outs))
    ref = torch.log_softmax(z.double(), 1)
    # 2^-15 of the best token's own, and a rounding
    bound = 2.0 ** -15 * -ref.max(1, keepdim=True).values + 2.0 ** -24 * ref.abs().max()
    assert ((outs[0][0] - ref.gather(1, tok.long())).abs() <= bound).all()
