"""Eviction: what its callers hand over. Nothing at all, from nothing and into nothing."""
from __future__ import annotations

import pytest
import torch

from paper_2601_04359_b200 import binding as pc
from tests.test_q4_cache import _ctx


@pytest.mark.gpu
@pytest.mark.parametrize("room", [0, 5])
def test_nothing_is_kept_of_nothing(room):
    ctx = _ctx("lumos", 1, 64)
    dst = pc.Q4Segment.empty(ctx, room, weight=True)
    dst.n_tokens = room
    sel = pc.pc_q4_evict(ctx, pc.Q4Segment.empty(ctx, 0, t_shift=3), 5, 2, dst, delta_t=4)
    assert dst.n_tokens == 0 and dst.t_shift == 7 and sel.dtype == torch.int32 and sel.is_cuda
    for weight in (None, torch.empty(0, device="cuda")):
        to = pc.Segment(torch.empty(room, 8, 128, dtype=torch.bfloat16, device="cuda"), torch.empty(room, 8, 128, dtype=torch.bfloat16, device="cuda"),
                        torch.empty(room, 4, dtype=torch.int32, device="cuda"), room) if room else pc.Segment.empty()
        sel = pc.pc_evict(ctx, pc.Segment.empty(), weight, 5, 2, to)
        assert to.n_tokens == 0 and sel.is_cuda
    assert pc.pc_poll_status(ctx) == pc.PC_OK
