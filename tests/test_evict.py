"""Eviction by accumulated attention weight, in 16 bits and in four, against a sort."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from paper_2601_04359_b200 import binding as pc
from tests import q4_reference as ref
from tests.test_q4_cache import _ctx, _refused, _rows

pytestmark = pytest.mark.gpu


def _weights(rng, n, kind):
    if kind == "spread":
        return np.exp(3 * rng.standard_normal(n)).astype(np.float32) / n
    if kind == "ties":
        return rng.integers(0, 5, n).astype(np.float32)
    if kind == "zeros":
        return np.where(rng.random(n) < 0.5, 0.0, -0.0).astype(np.float32)
    if kind == "close":                                   # differ in the last bits only
        return (1.0 + rng.integers(0, 64, n) * 2.0 ** -23).astype(np.float32)
    return np.where(rng.random(n) < 0.3, -1.0, 1.0).astype(np.float32) * np.float32(1e-40) * rng.integers(0, 9, n).astype(np.float32)


@pytest.mark.parametrize("kind", ["spread", "ties", "zeros", "close", "signs"])
@pytest.mark.parametrize("n,keep,recent", [(1, 1, 0), (5, 2, 1), (100, 99, 0), (100, 40, 40), (1000, 300, 135), (4097, 1, 0), (8193, 4000, 77), (9001, 9000, 5),
                                           (40000, 6048, 1008)])
def test_selection_matches_a_sort(kind, n, keep, recent):
    rng = np.random.default_rng(n + keep)
    ctx = _ctx("tiny_f32", 1, 64)
    w = _weights(rng, n, kind)
    k = torch.arange(n, device="cuda", dtype=torch.float32)[:, None, None].expand(n, 2, 64).contiguous()
    pos = torch.arange(4 * n, dtype=torch.int32, device="cuda").view(n, 4)
    src = pc.Segment(k, -k, pos, n)
    weight = torch.from_numpy(w).cuda()
    for valid in (None, rng.random(n) < 0.6):
        dst = pc.Segment(torch.full((keep, 2, 64), -7.0, device="cuda"), torch.full((keep, 2, 64), -7.0, device="cuda"),
                         torch.zeros(keep, 4, dtype=torch.int32, device="cuda"), 0)
        dw = torch.full((keep,), -7.0, device="cuda")
        v = None if valid is None else torch.from_numpy(valid.astype(np.uint8)).cuda()
        sel = pc.pc_evict(ctx, src, weight, keep, recent, dst, dw, delta_t=3, valid=v)
        assert pc.pc_poll_status(ctx) == pc.PC_OK
        want = ref.evict(w, keep, recent, valid)
        assert np.array_equal(sel.cpu().numpy(), want)
        at = torch.from_numpy(want).long().cuda()
        assert torch.equal(dst.k, src.k[at]) and torch.equal(dst.v, src.v[at]) and dst.n_tokens == keep
        assert torch.equal(dw.view(torch.int32), weight[at].view(torch.int32))
        assert torch.equal(dst.pos, src.pos[at] - torch.tensor([3, 0, 0, 0], dtype=torch.int32, device="cuda"))


@pytest.mark.parametrize("n", [300_001, 1_000_000])
def test_histories_longer_than_shared_memory(n):
    rng = np.random.default_rng(n)
    ctx = _ctx("tiny_f32", 1, 64)
    w = _weights(rng, n, "spread")
    k = torch.zeros(n, 2, 64, device="cuda")
    k[:, 0, 0] = torch.arange(n, device="cuda")
    src = pc.Segment(k, k, torch.zeros(n, 4, dtype=torch.int32, device="cuda"), n)
    keep, recent = n // 3, 1000
    dst = pc.Segment(k.new_empty(keep, 2, 64), k.new_empty(keep, 2, 64), torch.empty(keep, 4, dtype=torch.int32, device="cuda"), 0)
    sel = pc.pc_evict(ctx, src, torch.from_numpy(w).cuda(), keep, recent, dst)
    want = ref.evict(w, keep, recent)
    assert np.array_equal(sel.cpu().numpy(), want) and np.array_equal(dst.k[:, 0, 0].cpu().numpy().astype(np.int64), want)


@pytest.mark.parametrize("shape", ["lumos", "one", "small", "tiny_f32"])
@pytest.mark.parametrize("n,keep,recent,delta", [(200, 60, 20, 4), (64, 64, 0, 8), (64, 100, 10, 0), (10, 0, 0, 0), (12000, 3000, 1000, 4)])
def test_evicting_four_bit_rows(shape, n, keep, recent, delta):
    rng = np.random.default_rng(n)
    ctx = _ctx(shape, 1, 64)
    src, pos = _rows(rng, shape, n)
    seg = pc.Q4Segment.empty(ctx, n + 3, t_shift=12, weight=True)
    pc.pc_q4_store(ctx, src, seg)
    w = _weights(rng, n + 3, "ties")
    seg.weight.copy_(torch.from_numpy(w))
    dst = pc.Q4Segment.empty(ctx, max(keep, 1), weight=True)
    sel = pc.pc_q4_evict(ctx, seg, keep, recent, dst, delta_t=delta)
    assert pc.pc_poll_status(ctx) == pc.PC_OK
    kept = min(n, keep)
    want = ref.evict(w[:n], keep, recent)
    assert dst.n_tokens == kept == len(want) and dst.t_shift == 12 + delta
    assert np.array_equal(sel.cpu().numpy()[:kept], want)
    at = torch.from_numpy(want).long().cuda()
    assert torch.equal(dst.rows[:kept], seg.rows[at]) and torch.equal(dst.weight[:kept], seg.weight[at])
    assert np.array_equal(dst.pos.cpu().numpy()[:kept], pos[want] - np.array([delta, 0, 0, 0]))
    if kept:
        # the rebase has left the keys where they were: what comes back is what was there
        a = pc.Segment(torch.empty_like(src.k), torch.empty_like(src.v), torch.empty_like(src.pos), 0)
        b = pc.Segment(torch.empty_like(src.k[:kept]), torch.empty_like(src.v[:kept]), torch.empty_like(src.pos[:kept]), 0)
        pc.pc_q4_load(ctx, seg, 0, n, a)
        pc.pc_q4_load(ctx, dst, 0, kept, b)
        assert torch.equal(a.k[at], b.k) and torch.equal(a.v[at], b.v)


def test_accumulated_masses():
    ctx = _ctx("lumos", 1, 64)
    m, w = torch.rand(1001, device="cuda"), torch.rand(1003, device="cuda")
    want = w.double()
    want[:1001] = 0.75 * want[:1001] + 2.0 * m.double()
    pc.pc_accumulate(ctx, m, w, 0.75, 2.0)
    assert pc.pc_poll_status(ctx) == pc.PC_OK
    assert (w.double() - want).abs().max() <= 2.0 ** -22 * 3
    pc.pc_accumulate(ctx, m[1:], w[2:], 1.0, 0.0)        # 4-byte alignment is enough
    assert (w.double() - want).abs().max() <= 2.0 ** -22 * 3


def test_nan_weights_are_recorded_unless_masked():
    ctx = _ctx("tiny_f32", 1, 64)
    src, _ = _rows(np.random.default_rng(0), "tiny_f32", 20)
    w = torch.rand(20, device="cuda")
    w[3] = float("nan")
    dst = pc.Segment(torch.empty_like(src.k), torch.empty_like(src.v), torch.empty_like(src.pos), 0)
    pc.pc_evict(ctx, src, w, 10, 0, dst)
    assert pc.pc_poll_status(ctx) == pc.PC_ERR_INVALID_ARG
    valid = torch.ones(20, dtype=torch.uint8, device="cuda")
    valid[3] = 0
    sel = pc.pc_evict(ctx, src, w, 10, 0, dst, valid=valid)
    assert pc.pc_poll_status(ctx) == pc.PC_OK and 3 not in sel.cpu().tolist()


def test_refusals():
    ctx = _ctx("lumos", 1, 64)
    src, _ = _rows(np.random.default_rng(1), "lumos", 30)
    seg = pc.Q4Segment.empty(ctx, 30, weight=True)
    pc.pc_q4_store(ctx, src, seg)
    dst = pc.Q4Segment.empty(ctx, 10, weight=True)
    _refused(pc.PC_ERR_INVALID_ARG, pc.pc_q4_evict, ctx, seg, 10, 11, dst)
    _refused(pc.PC_ERR_INVALID_ARG, pc.pc_q4_evict, ctx, seg, -1, 0, dst)
    _refused(pc.PC_ERR_CAPACITY, pc.pc_q4_evict, ctx, seg, 11, 0, dst)
    _refused(pc.PC_ERR_INVALID_ARG, pc.pc_q4_evict, ctx, seg, 10, 0, dst, delta_t=-1)    # there is no shift to take back
    _refused(pc.PC_ERR_INVALID_ARG, pc.pc_q4_evict, ctx, seg, 10, 0, pc.Q4Segment(seg.rows[20:], dst.pos, dst.weight, 0))
    seg.weight = None
    _refused(pc.PC_ERR_INVALID_ARG, pc.pc_q4_evict, ctx, seg, 10, 0, dst)
    w = torch.rand(30, device="cuda")
    to = pc.Segment(torch.empty_like(src.k[:10]), torch.empty_like(src.v[:10]), torch.empty_like(src.pos[:10]), 0)
    _refused(pc.PC_ERR_INVALID_ARG, pc.pc_evict, ctx, src, w, 10, 0, pc.Segment(src.v[:10], to.v, to.pos, 0))
    _refused(pc.PC_ERR_CAPACITY, pc.pc_evict, ctx, src, w, 12, 0, to)
    _refused(pc.PC_ERR_INVALID_ARG, pc.pc_evict, ctx, src, w, 10, 0, to, w[20:])
    assert to.n_tokens == 0 and dst.n_tokens == 0 and pc.pc_poll_status(ctx) == pc.PC_OK


@pytest.mark.parametrize("n", [300, 9000, 40000])
@pytest.mark.parametrize("near,same", [(1, 1), (2, 1), (2, 2), (31, 3), (32, 1), (32, 32), (33, 5), (40, 1)])
def test_few_tokens_around_the_last_that_stays(n, near, same):
    """`near` weights that share all but their last bits, `same` of them equal, the last that stays among them."""
    rng = np.random.default_rng(n + near + same)
    ctx = _ctx("tiny_f32", 1, 64)
    above = n // 5
    w = np.concatenate([2 + rng.random(above), 1 + 2.0 ** -23 * np.maximum(np.arange(near), same - 1), 0.5 * rng.random(n - above - near)]).astype(np.float32)
    w = w[rng.permutation(n)]
    k = torch.arange(n, device="cuda", dtype=torch.float32)[:, None, None].expand(n, 2, 64).contiguous()
    src = pc.Segment(k, k, torch.zeros(n, 4, dtype=torch.int32, device="cuda"), n)
    masked = np.ones(n, bool)
    masked[rng.permutation(n)[:near]] = False
    for keep, valid in ((above + 1, None), (above + near // 2, None), (above + near, None), (n - near + near // 2, masked)):
        dst = pc.Segment(k.new_empty(keep, 2, 64), k.new_empty(keep, 2, 64), torch.empty(keep, 4, dtype=torch.int32, device="cuda"), 0)
        v = None if valid is None else torch.from_numpy(valid.astype(np.uint8)).cuda()
        sel = pc.pc_evict(ctx, src, torch.from_numpy(w).cuda(), keep, 0, dst, valid=v)
        assert pc.pc_poll_status(ctx) == pc.PC_OK
        want = ref.evict(w, keep, 0, valid)
        assert np.array_equal(sel.cpu().numpy(), want) and np.array_equal(dst.k[:, 0, 0].cpu().numpy().astype(np.int64), want)
