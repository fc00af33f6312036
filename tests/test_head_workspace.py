"""Workspace of the head's training operators: what a call holds of its rows at
a time is bounded, whichever of rows, channels, symbols and entries is large.
CPU only."""
import os

import pytest
import torch

import paper_2503_12382_amd as reno

pytestmark = pytest.mark.skipif(not os.path.exists(reno.LIB_PATH),
                                reason="libreno.so not built (run __graft_entry__.build())")
TYPES = [torch.float32, torch.bfloat16, torch.float16]


@pytest.mark.parametrize("grad", [False, True])
@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("N,C,V,k", [(4 << 20, 2048, 16, 1), (4 << 20, 16384, 16, 1), (1 << 22, 200, 16, 128),
                                     (1 << 20, 300, 300, 64), (1 << 20, 64, 1 << 20, 1), (2 ** 31 - 1, 200, 16, 1)])
def test_pieces_are_bounded(N, C, V, k, dt, grad):
    up = (C + 63) // 64 * 64, (V + 255) // 256 * 256
    whole = N * (8 * k + 5)                            # every row's targets
    weights = 3 * C * up[1] * 2 + 2 * up[1] * 4        # packed weights, bias and its gradient's sums
    sums = C * V * 4 + (1 << 27)                       # sums of dw of several pieces; splits of k, 2^26 of each product
    copies = 1 << 31                                   # rows of h as planes, t of the targets
    logits = 10 << 27 if dt == torch.float32 else 6 << 28   # kept for the gradient: t, and dz as planes
    stats = 1 << 30                                    # maxima and sums of parts of 64 symbols, of 2^32 logits; sums over rows
    most = whole + weights + copies + stats + ((logits + sums) if grad else 0)
    assert reno.head_workspace(N, C, V, dt, k, grad) <= most


@pytest.mark.parametrize("dt", TYPES)
def test_a_few_rows_need_little(dt):
    assert reno.head_workspace(256, 64, 1000, dt, 1, False) < 4 << 20
    assert reno.head_workspace(1, 2048, 65536, dt, 1, False) < 1 << 20
