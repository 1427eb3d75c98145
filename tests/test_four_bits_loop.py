"""The generation loop over the 4-bit cache: frames, text tokens, weights and evictions together; and waits that run out in its attention."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from paper_2601_04359_b200 import binding as pc
from paper_2601_04359_b200 import four_bits
from tests.test_q4_cache import Case, _np, _rows

pytestmark = pytest.mark.gpu


def test_the_loop_keeps_its_cache_and_its_answers():
    r = four_bits.generate(frames=6, tokens=3, budget=300, grid=(9, 15), heads=(24, 8), n_text=37, reps=2)
    step = 9 * 15 + 3
    assert r["evictions"] == 3 and r["t_shift"] == 3 * four_bits.T_STEP
    assert r["history"] == 300 + step
    # bf16 attention of the same tokens: its own roundings (the query, keys, probabilities and values in bf16)
    assert r["off_16bit"] <= 2e-2 * 8
    # every token of text pays one unit of attention, of which anchors take a part and evictions and decay more
    assert 0.0 < r["weight"] <= 18.0
    assert r["bytes_16bit"] / r["bytes_4bit"] == 3.2


@pytest.mark.parametrize("n_hist,n_q,frames", [(40, 1, False), (3000, 1, False), (3000, 5, False), (300, 130, True)])
def test_a_wait_that_runs_out_is_reported_and_the_workspace_survives(n_hist, n_q, frames):
    """The limit is two milliseconds and the first barrier of every CTA is told to expect sixteen bytes more than are ever sent."""
    c = Case("lumos", 33, n_hist, n_q, frames=frames)
    good, good_lse = pc.pc_q4_attend(c.work, c.cache, c.q, c.q_pos, want_lse=True)
    assert pc.pc_poll_status(c.ctx) == pc.PC_OK
    pc.pc_set_wait_limit_us(c.ctx, 2000)
    pc.pc_test_expect_extra_bytes(c.ctx, 16)
    pc.pc_q4_attend(c.work, c.cache, c.q, c.q_pos)
    assert pc.pc_poll_status(c.ctx) == pc.PC_ERR_TIMEOUT
    assert pc.pc_poll_status(c.ctx) == pc.PC_OK
    pc.pc_test_expect_extra_bytes(c.ctx, 0)
    pc.pc_set_wait_limit_us(c.ctx, 0)
    again, lse = pc.pc_q4_attend(c.work, c.cache, c.q, c.q_pos, want_lse=True)
    assert pc.pc_poll_status(c.ctx) == pc.PC_OK
    assert torch.equal(again, good) and torch.equal(lse, good_lse)


def test_sixteen_bit_calls_after_a_frame_over_four_bits():
    """A frame over the 4-bit cache uses the context's rotated-key scratch: what pc_attend_prepare fixed is dropped, masses are not on offer,
    and a 16-bit call behind it is right."""
    c = Case("lumos", 20, 200, 130, frames=True)
    h = c.hist
    seg = pc.Segment(torch.empty(200, 8, 128, dtype=torch.bfloat16, device="cuda"), torch.empty(200, 8, 128, dtype=torch.bfloat16, device="cuda"),
                     torch.empty(200, 4, dtype=torch.int32, device="cuda"), 0)
    pc.pc_q4_load(c.ctx, h, 0, 200, seg)
    cache = pc.Cache(pc.Segment.empty(), seg, [200])
    pc.pc_attend_prepare(c.ctx, cache)
    want, lse = pc.pc_attend_prepared(c.ctx, c.q, c.q_pos, want_lse=True)
    out = pc.pc_q4_attend(c.work, pc.Q4Cache(pc.Q4Segment.empty(c.ctx, 0), h), c.q, c.q_pos)
    with pytest.raises(pc.PackCacheError) as e:
        pc.pc_attend_prepared(c.ctx, c.q, c.q_pos)
    assert e.value.status == pc.PC_ERR_INVALID_ARG
    with pytest.raises(pc.PackCacheError) as e:
        pc.pc_attend_mass(c.ctx, lse, 200)
    assert e.value.status == pc.PC_ERR_INVALID_ARG
    again = pc.pc_attend_frame(c.ctx, cache, None, c.q, c.q_pos)
    assert pc.pc_poll_status(c.ctx) == pc.PC_OK
    assert torch.equal(again, want)
    assert abs(_np(out) - _np(want)).max() <= 2e-2 * max(1.0, abs(_np(want)).max())


@pytest.mark.parametrize("n_q,frames", [(1, False), (40, True)])
def test_calls_replay_from_a_cuda_graph(n_q, frames):
    c = Case("lumos", 96, 384, n_q, shift=8, weight=True, frames=frames)
    raw = _rows(np.random.default_rng(3), "lumos", 64)[0]
    out, lse = torch.empty_like(c.q), torch.empty(n_q, c.q.shape[1], device="cuda")
    dst = pc.Q4Segment.empty(c.ctx, 200, weight=True)
    sel = torch.empty(200, dtype=torch.int32, device="cuda")

    def calls():
        pc.pc_q4_store(c.ctx, raw, c.hist, at=320)
        pc.pc_q4_attend(c.work, c.cache, c.q, c.q_pos, weigh=None if frames else (0.5, 1.0), out=out, lse=lse)
        pc.pc_q4_evict(c.ctx, c.hist, 200, 50, dst, delta_t=4, sel_idx=sel)

    def result():
        torch.cuda.synchronize()
        return [x.clone() for x in (out, lse, dst.rows, dst.pos, dst.weight, sel)]

    start = torch.rand(384, device="cuda")
    s, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        calls()
        with torch.cuda.graph(graph, stream=s):
            calls()
    torch.cuda.synchronize()
    for scale in (1.0, 0.5):                                 # inputs changed in place between replays
        c.q.mul_(scale)
        raw.k.mul_(scale)
        c.hist.weight.copy_(start)
        calls()
        want = result()
        for x in (out, lse, dst.rows, dst.weight, sel):
            x.zero_()
        c.hist.weight.copy_(start)
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(result(), want))
    assert pc.pc_poll_status(c.ctx) == pc.PC_OK
