"""The 4-bit cache: rows written and read back, attention over it with masks and weights, against fp64 restatements.

Tolerances.  A logit of the kernel is off by what its sums round: the query's two fp16 parts hold 22 bits, products with codes are
exact, and no more than 48 additions in fp32, each 2^-23 of a partial sum that is at most S = sum |q| (step code + |low|) / sqrt(d), so
delta <= (48 * 2^-23 + 2^-21) S.  Probabilities are then off by 2 delta + 2^-18 relative (exponential, sums, normaliser).  Outputs add the
roundings of probability times step: two to fp16 in bf16 contexts (2^-10 in all, of sum p (step code + |low|)), 2^-20 in fp32 ones, where the
probability and the product are each held in parts; and half a unit of the output's type."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from paper_2601_04359_b200 import binding as pc
from tests import q4_reference as ref

pytestmark = pytest.mark.gpu

MAX_POS = (600, 400, 400)
SHAPES = {"lumos": (24, 8, 128, "bf16"), "gqa4": (32, 8, 128, "bf16"), "mha": (8, 8, 128, "bf16"), "wide": (24, 12, 128, "bf16"),
          "one": (7, 1, 128, "bf16"), "many": (20, 20, 128, "bf16"), "small": (4, 2, 64, "bf16"), "odd64": (9, 3, 64, "bf16"),
          "tiny_f32": (4, 2, 64, "f32"), "lumos_f32": (24, 8, 128, "f32")}


def _t(x, dtype):
    t = torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).cuda()
    return t.to(torch.bfloat16) if dtype == "bf16" else t


def _np(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def _pos(rng, n):
    p = np.stack([rng.integers(0, 300, n), rng.integers(0, 400, n), rng.integers(0, 400, n), np.arange(n)], 1).astype(np.int32)
    return p


def _ctx(shape, max_q, max_keys):
    hq, hkv, d, dtype = SHAPES[shape]
    return pc.Context(hq, hkv, d, pc.PC_BF16 if dtype == "bf16" else pc.PC_F32, 10000.0, MAX_POS, max_q, max_keys)


def _rows(rng, shape, n, scale=1.0):
    hq, hkv, d, dtype = SHAPES[shape]
    k, v = (_t(rng.standard_normal((n, hkv, d)) * scale, dtype) for _ in range(2))
    bias = np.zeros((hkv, d), np.float32)
    bias.reshape(-1)[rng.permutation(hkv * d)[: hkv * d // 50 + 1]] = 4.0 * scale
    k = (k.float() + torch.from_numpy(bias).cuda()).to(k.dtype)
    pos = _pos(rng, n)
    return pc.Segment(k, v, torch.from_numpy(pos).cuda(), n), pos


# ---------------------------------------------------------------------------------------------------------------------
# store and load
# ---------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("shape", list(SHAPES))
@pytest.mark.parametrize("n,at,shift", [(1, 0, 0), (67, 3, 40), (130, 0, 0)])
def test_store_and_load(shape, n, at, shift):
    hq, hkv, d, dtype = SHAPES[shape]
    rng = np.random.default_rng(n + hq)
    ctx = _ctx(shape, 1, 256)
    src, pos = _rows(rng, shape, n)
    seg = pc.Q4Segment.empty(ctx, at + n + 2, t_shift=shift, weight=True)
    seg.rows.fill_(0xA5)
    seg.weight.fill_(7.0)
    seg.n_tokens = at
    pc.pc_q4_store(ctx, src, seg)
    assert pc.pc_poll_status(ctx) == pc.PC_OK
    assert seg.n_tokens == at + n
    rows = seg.rows.cpu().numpy()
    assert (rows[:at] == 0xA5).all() and (rows[at + n:] == 0xA5).all()
    w = seg.weight.cpu().numpy()
    assert (w[at:at + n] == 0).all() and (w[:at] == 7).all() and (w[at + n:] == 7).all()
    assert np.array_equal(seg.pos.cpu().numpy()[at:at + n], pos)
    kq, vq = ref.decode(rows[at:at + n], d)
    want_k, want_v = ref.quantise(ref.turn(_np(src.k), pos, shift)), ref.quantise(_np(src.v))
    for got, want, x in ((kq, want_k, ref.turn(_np(src.k), pos, shift)), (vq, want_v, _np(src.v))):
        # fp32 arithmetic moves a value by less than 2^-21 of its group's largest: lows and steps may round the other way, codes at ties
        big = np.abs(x).reshape(n, hkv, -1, 32).max(-1)
        assert (np.abs(got[2] - want[2]) <= 2.0 ** -10 * big).all()
        assert (np.abs(got[1] - want[1]) <= 2.0 ** -10 * np.maximum(want[1], big / 15)).all()
        assert np.abs(got[0] - want[0]).max() <= 1 and (got[0] != want[0]).mean() <= 1e-3
        assert (np.abs(ref.values(got) - x).reshape(n, hkv, -1, 32) <= (0.5 + 2.0 ** -6) * want[1][..., None] + 2.0 ** -10 * big[..., None]).all()
    back = pc.Segment(torch.empty_like(src.k), torch.empty_like(src.v), torch.empty_like(src.pos), 0)
    pc.pc_q4_load(ctx, seg, at, n, back)
    assert pc.pc_poll_status(ctx) == pc.PC_OK and back.n_tokens == n
    unit = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -22
    tol = lambda x: unit * np.abs(x) + 2.0 ** -21 * np.abs(x).max()                                 # noqa: E731
    v = ref.values(vq)
    k = ref.turn(ref.values(kq), pos, shift, -1.0)
    assert (np.abs(_np(back.v) - v) <= tol(v)).all()
    assert (np.abs(_np(back.k) - k) <= tol(k)).all()
    assert np.array_equal(back.pos.cpu().numpy(), pos)


def test_store_of_what_half_precision_cannot_hold():
    ctx = _ctx("tiny_f32", 1, 64)
    src, pos = _rows(np.random.default_rng(0), "tiny_f32", 4)
    src.pos.zero_()
    src.v[0, 0, 3] = float("nan")
    src.v[1, 1, 40] = float("inf")
    src.v[2, 0, 8] = -1e30
    src.v[3, 0, :32] = 2.5
    src.v[3, 0, 32:] = 1e-7
    seg = pc.Q4Segment.empty(ctx, 4)
    pc.pc_q4_store(ctx, src, seg)
    assert pc.pc_poll_status(ctx) == pc.PC_ERR_INVALID_ARG
    v = ref.values(ref.decode(seg.rows.cpu().numpy(), 64)[1])
    x = _np(src.v)
    x[0, 0, 3], x[1, 1, 40], x[2, 0, 8] = 0.0, 65504.0, -65504.0
    want = ref.values(ref.quantise(x))
    assert np.isfinite(v).all() and (np.abs(v - want) <= 2.0 ** -9 * np.maximum(1, np.abs(want))).all()
    assert (v[3, 0, :32] == 2.5).all() and (np.abs(v[3, 0, 32:] - 1e-7) <= 2.0 ** -25).all()


def test_a_whole_clip_in_pieces_is_the_clip():
    """Rows written one by one, in pieces and at once are the same bytes."""
    ctx = _ctx("wide", 1, 512)
    src, _ = _rows(np.random.default_rng(5), "wide", 203)
    whole, pieces = pc.Q4Segment.empty(ctx, 203), pc.Q4Segment.empty(ctx, 203)
    pc.pc_q4_store(ctx, src, whole)
    for a, b in ((0, 1), (1, 2), (2, 130), (130, 203)):
        pc.pc_q4_store(ctx, pc.Segment(src.k[a:b], src.v[a:b], src.pos[a:b], b - a), pieces)
    assert torch.equal(whole.rows, pieces.rows) and torch.equal(whole.pos, pieces.pos) and pieces.n_tokens == 203


# ---------------------------------------------------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------------------------------------------------
class Case:
    def __init__(self, shape, n_anchor, n_hist, n_q, shift=0, seed=0, weight=False, scale=1.0, frames=False, max_tokens=0, max_q=0, q_scale=1.0):
        hq, hkv, d, dtype = SHAPES[shape]
        rng = np.random.default_rng(seed + 17 * n_hist + n_q)
        self.shape, self.rng, self.d, self.dtype = shape, rng, d, dtype
        self.ctx = _ctx(shape, max_q or n_q, max(n_anchor + n_hist, 1))
        self.anchors, self.hist = pc.Q4Segment.empty(self.ctx, n_anchor), pc.Q4Segment.empty(self.ctx, n_hist, t_shift=shift, weight=weight)
        for seg, n in ((self.anchors, n_anchor), (self.hist, n_hist)):
            if n:
                pc.pc_q4_store(self.ctx, _rows(rng, shape, n, scale)[0], seg)
        self.cache = pc.Q4Cache(self.anchors, self.hist)
        self.q, self.q_pos = _t(rng.standard_normal((n_q, hq, d)) * q_scale, dtype), torch.from_numpy(_pos(rng, n_q)).cuda()
        self.work = pc.Q4Work(self.ctx, max_tokens or max(n_anchor + n_hist, 1), frames=frames, weigh=weight)

    def parts(self):
        out = []
        for seg in (self.anchors, self.hist):
            rows = seg.rows[:seg.n_tokens].cpu().numpy() if seg.rows is not None else np.zeros((0, SHAPES[self.shape][1] * 5 * self.d // 4), np.uint8)
            kq, vq = ref.decode(rows, self.d)
            out.append((kq, vq, seg.t_shift))
        return out

    def check(self, valid=None, weigh=None, coarse=0.0, parts=None):
        before = _np(self.hist.weight) if weigh else None
        v = torch.from_numpy(np.ascontiguousarray(valid, dtype=np.uint8)).cuda() if valid is not None else None
        out = torch.full_like(self.q, float("nan"))
        out, lse = pc.pc_q4_attend(self.work, self.cache, self.q, self.q_pos, valid=v, weigh=weigh, out=out, want_lse=True)
        assert pc.pc_poll_status(self.ctx) == pc.PC_OK
        want, want_lse, mass, mag_l, mag_v = ref.attend(_np(self.q), self.q_pos.cpu().numpy(), parts or self.parts(), valid)
        delta = (48 * 2.0 ** -23 + 2.0 ** -21) * mag_l + coarse
        p_off = 2 * delta + 2.0 ** -18
        f32 = self.dtype == "f32"
        tol = (p_off + (2.0 ** -20 if f32 else 2.0 ** -10))[..., None] * mag_v + (2.0 ** -23 if f32 else 2.0 ** -8) * np.abs(want) + coarse * mag_v
        got = _np(out)
        assert np.isfinite(got).all()
        assert (np.abs(got - want) <= tol).all(), (np.abs(got - want) / tol).max()
        got_lse = _np(lse)
        empty = ~np.isfinite(want_lse)
        assert (got_lse[empty] == -np.inf).all() and (got[empty] == 0).all()
        assert (np.abs(got_lse - want_lse)[~empty] <= (delta + 2.0 ** -20 * (1 + np.abs(np.where(empty, 0, want_lse))))[~empty]).all()
        if weigh:
            n_hist = self.hist.n_tokens
            want_w = np.float32(weigh[0]) * before[:n_hist] + weigh[1] * mass[len(mass) - n_hist:]
            tol_w = weigh[1] * mass[len(mass) - n_hist:] * (p_off.max() + 2.0 ** -18) + 2.0 ** -22 * np.abs(want_w)
            assert (np.abs(_np(self.hist.weight)[:n_hist] - want_w) <= tol_w).all()
        return out, lse


@pytest.mark.parametrize("shape", list(SHAPES))
@pytest.mark.parametrize("n_anchor,n_hist,n_q", [(0, 1, 1), (1, 0, 1), (37, 203, 1), (5, 530, 2), (96, 384, 5)])
def test_attention(shape, n_anchor, n_hist, n_q):
    Case(shape, n_anchor, n_hist, n_q, shift=24).check()


@pytest.mark.parametrize("n", [15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 129, 1000])
def test_lengths_around_the_tiles(n):
    Case("lumos", 0, n, 1, seed=n).check()
    Case("lumos", n, 3, 3, seed=n, shift=8).check()


@pytest.mark.parametrize("shape,n_q", [("lumos", 2), ("lumos", 3), ("lumos", 6), ("lumos", 9), ("lumos", 40), ("one", 16), ("many", 11), ("odd64", 30), ("tiny_f32", 64)])
def test_blocks_of_query_rows(shape, n_q):
    Case(shape, 21, 150, n_q, shift=4).check()


@pytest.mark.parametrize("shape", ["lumos", "one", "tiny_f32", "lumos_f32"])
def test_masks(shape):
    c = Case(shape, 20, 301, 2, weight=True)
    for valid in (c.rng.random(301) < 0.7, np.arange(301) < 5, np.arange(301) >= 290, np.zeros(301), np.ones(301), np.arange(301) % 16 == 7):
        c.check(valid, weigh=(0.9, 2.0))
    c = Case(shape, 0, 75, 3, weight=True)
    c.hist.weight.copy_(torch.rand(75))
    c.check(np.zeros(75), weigh=(0.5, 1.0))               # nothing is left: out 0, lse -infinity, weights only decay
    c.check(np.arange(75) == 74, weigh=(0.5, 1.0))


@pytest.mark.parametrize("shape", ["lumos", "small", "tiny_f32"])
@pytest.mark.parametrize("byte", [0xFF, 0x7C, 0xFB])     # steps and lows that are NaN, large and infinite
def test_masked_rows_may_hold_anything(shape, byte):
    n = 147
    c = Case(shape, 9, n, 2, weight=True)
    valid = c.rng.random(n) < 0.5
    parts = c.parts()
    c.hist.rows[torch.from_numpy(~valid).cuda()] = byte
    if byte == 0x7C:
        c.hist.rows[torch.from_numpy(~valid).cuda(), 0::2] = 0          # 0x7c00: infinity
    c.check(valid, weigh=(1.0, 1.0), parts=parts)


def test_rows_behind_the_tokens_in_use_are_not_read_into_results():
    c = Case("lumos", 33, 70, 1)
    for seg in (c.anchors, c.hist):
        seg.rows[-6:] = 0xFF
        seg.n_tokens -= 6
    c.check()


@pytest.mark.parametrize("shape", ["lumos", "gqa4", "odd64", "tiny_f32"])
def test_weights(shape):
    c = Case(shape, 40, 333, 4, weight=True)
    c.hist.weight.copy_(torch.rand(333))
    c.check(weigh=(0.98, 1.0))
    c.check(weigh=(0.0, 3.0))
    c.check(c.rng.random(333) < 0.5, weigh=(1.0, 4.0))


def test_weights_in_several_passes():
    """More logits than the workspace holds: the queries go in passes, the decay is taken once."""
    n, n_q = 12001, 90                                   # 24 heads x 12,001 tokens x 90 queries are 26 million logits
    c = Case("lumos", 8, n, n_q, weight=True)
    assert n * 24 * n_q > 16 << 20
    c.hist.weight.fill_(0.01)
    v = torch.ones(n, dtype=torch.uint8, device="cuda")
    out = pc.pc_q4_attend(c.work, c.cache, c.q, c.q_pos, valid=v, weigh=(0.5, 1.0))
    got = _np(c.hist.weight)
    # the same queries one by one
    w = torch.full((n,), 0.005, dtype=torch.float64, device="cuda")
    for i in range(n_q):
        c.hist.weight.zero_()
        one = pc.pc_q4_attend(c.work, c.cache, c.q[i:i + 1], c.q_pos[i:i + 1], weigh=(1.0, 1.0))
        w += c.hist.weight.double() / n_q
        assert torch.allclose(one.float(), out[i:i + 1].float(), rtol=2.0 ** -7, atol=2.0 ** -8)
    assert pc.pc_poll_status(c.ctx) == pc.PC_OK
    assert (np.abs(got - w.cpu().numpy()) <= 1e-4 * (got - 0.005) + 1e-8).all()


def test_large_and_small_queries_and_values():
    for q_scale, scale in ((1e-3, 1.0), (30.0, 1.0), (1.0, 1e-2), (1.0, 300.0 / 16)):
        Case("lumos", 10, 100, 2, q_scale=q_scale, scale=scale).check()
        Case("tiny_f32", 10, 100, 2, q_scale=q_scale, scale=scale).check()
    c = Case("lumos", 10, 100, 2)
    c.q.zero_()                                          # every key alike
    c.check()


def test_same_bits_again():
    c = Case("lumos", 100, 3000, 3, weight=True)
    a = pc.pc_q4_attend(c.work, c.cache, c.q, c.q_pos, weigh=(0.0, 1.0))
    wa = c.hist.weight.clone()
    for _ in range(3):
        b = pc.pc_q4_attend(c.work, c.cache, c.q, c.q_pos, weigh=(0.0, 1.0))
        assert torch.equal(a, b) and torch.equal(wa, c.hist.weight)


def test_on_another_stream():
    c = Case("lumos", 64, 2000, 1)
    want = pc.pc_q4_attend(c.work, c.cache, c.q, c.q_pos)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    out = torch.empty_like(want)
    with torch.cuda.stream(s):
        pc.pc_q4_attend(c.work, c.cache, c.q, c.q_pos, out=out)
    s.synchronize()
    assert torch.equal(out, want)


@pytest.mark.parametrize("shape,n_q,shift", [("lumos", 100, 0), ("lumos", 130, 40), ("mha", 200, 12), ("gqa4", 40, 8)])
def test_frames_on_the_tensor_core_kernel(shape, n_q, shift):
    """Keys, values and probabilities in fp16 (2^-12 of each, at most), queries in two parts: a logit is off by 2^-12 of sum |q k| / sqrt(d) and what fp32
    sums round, an output by twice that and two more roundings of sum p |v|, and the rounding to bf16."""
    c = Case(shape, 70, 300, n_q, shift=shift, frames=True)
    want, want_lse, _, mag_l, mag_v = ref.attend(_np(c.q), c.q_pos.cpu().numpy(), c.parts())
    out, lse = pc.pc_q4_attend(c.work, c.cache, c.q, c.q_pos, want_lse=True)
    assert pc.pc_poll_status(c.ctx) == pc.PC_OK
    assert np.abs(_np(lse) - want_lse).max() <= 2e-2 and np.abs(_np(out) - want).max() <= 2e-2 * max(1.0, np.abs(want).max())
    delta = (2.0 ** -12 + 48 * 2.0 ** -23) * mag_l
    assert (np.abs(_np(lse) - want_lse) <= delta + 2.0 ** -20 * (1 + np.abs(want_lse))).all()
    assert (np.abs(_np(out) - want) <= (2 * delta + 2.0 ** -11)[..., None] * mag_v + 2.0 ** -8 * np.abs(want)).all()
    slow = pc.Q4Work(c.ctx, 370)
    rows = _np(pc.pc_q4_attend(slow, c.cache, c.q, c.q_pos))
    assert np.abs(rows - want).max() <= 2e-2 * max(1.0, np.abs(want).max())


def test_a_long_cache():
    """Offsets that pass 32 bits: rows of 20 KV heads are 3,200 bytes, 1.4 million of them 4.5 GB.  All but the last tokens are masked,
    and the answer is that of the last tokens alone."""
    hq, hkv, d, dtype = SHAPES["many"]
    n, last = 1_400_003, 70
    ctx = pc.Context(hq, hkv, d, pc.PC_BF16, 10000.0, MAX_POS, 1, 256)
    rng = np.random.default_rng(3)
    seg = pc.Q4Segment.empty(ctx, n, weight=True)
    seg.rows.zero_()
    seg.pos.zero_()
    seg.n_tokens = n - last
    src, _ = _rows(rng, "many", last)
    pc.pc_q4_store(ctx, src, seg)
    assert seg.n_tokens == n
    alone = pc.Q4Segment.empty(ctx, last)
    pc.pc_q4_store(ctx, src, alone)
    assert torch.equal(alone.rows, seg.rows[n - last:])
    q, q_pos = _t(rng.standard_normal((1, hq, d)), "bf16"), torch.from_numpy(_pos(rng, 1)).cuda()
    none = pc.Q4Segment.empty(ctx, 0)
    work = pc.Q4Work(ctx, n, weigh=True)
    valid = torch.zeros(n, dtype=torch.uint8, device="cuda")
    valid[n - last:] = 1
    out = pc.pc_q4_attend(work, pc.Q4Cache(none, seg), q, q_pos, valid=valid, weigh=(1.0, 1.0))
    want = pc.pc_q4_attend(work, pc.Q4Cache(none, alone), q, q_pos)
    assert pc.pc_poll_status(ctx) == pc.PC_OK
    assert torch.allclose(out.float(), want.float(), rtol=2.0 ** -7, atol=2.0 ** -9)
    w = seg.weight
    assert (w[: n - last] == 0).all() and abs(float(w.sum()) - 1.0) <= 1e-4
    back = pc.Segment(torch.empty_like(src.k), torch.empty_like(src.v), torch.empty_like(src.pos), 0)
    pc.pc_q4_load(ctx, seg, n - last, last, back)
    assert (back.v.float() - src.v.float()).abs().max() <= 0.5
    dst = pc.Q4Segment.empty(ctx, 100, weight=True)
    sel = pc.pc_q4_evict(ctx, seg, 100, 0, dst)
    assert pc.pc_poll_status(ctx) == pc.PC_OK
    assert sel.cpu().tolist() == list(range(30)) + list(range(n - last, n))
    assert torch.equal(dst.rows[30:], seg.rows[n - last:])


# ---------------------------------------------------------------------------------------------------------------------
# refusals
# ---------------------------------------------------------------------------------------------------------------------
def _refused(status, f, *a, **k):
    with pytest.raises(pc.PackCacheError) as e:
        f(*a, **k)
    assert e.value.status == status


def test_refusals():
    c = Case("lumos", 16, 40, 1, max_q=2)
    ctx, cache, q, q_pos, work = c.ctx, c.cache, c.q, c.q_pos, c.work
    src, _ = _rows(np.random.default_rng(1), "lumos", 8)
    small = pc.Q4Segment.empty(ctx, 4)
    _refused(pc.PC_ERR_CAPACITY, pc.pc_q4_store, ctx, src, small)
    _refused(pc.PC_ERR_INVALID_ARG, pc.pc_q4_store, ctx, src, small, 1)                   # a gap
    _refused(pc.PC_ERR_INVALID_ARG, pc.pc_q4_store, ctx, src, pc.Q4Segment.empty(ctx, 8, t_shift=-1))
    bad = pc.Q4Segment(torch.empty(8 * 1280 + 1, dtype=torch.uint8, device="cuda")[1:].view(8, 1280), small.pos, None, 0)
    _refused(pc.PC_ERR_INVALID_ARG, pc.pc_q4_store, ctx, src, bad)
    back = pc.Segment(src.k, src.v, src.pos, 0)
    _refused(pc.PC_ERR_INVALID_ARG, pc.pc_q4_load, ctx, c.hist, 38, 3, back)
    _refused(pc.PC_ERR_INVALID_ARG, pc.pc_q4_load, ctx, c.hist, -1, 3, back)
    _refused(pc.PC_ERR_CAPACITY, pc.pc_q4_load, ctx, c.hist, 0, 9, back)
    assert back.n_tokens == 0
    none = pc.Q4Segment.empty(ctx, 0)
    _refused(pc.PC_ERR_INVALID_ARG, pc.pc_q4_attend, work, pc.Q4Cache(none, none), q, q_pos)
    _refused(pc.PC_ERR_INVALID_ARG, pc.pc_q4_attend, work, cache, q, q_pos, weigh=(1.0, 1.0))     # no room for weights
    _refused(pc.PC_ERR_INVALID_ARG, pc.pc_q4_attend, pc.Q4Work(ctx, 56, weigh=True), cache, q, q_pos, weigh=(1.0, 1.0))   # no weights
    _refused(pc.PC_ERR_CAPACITY, pc.pc_q4_attend, pc.Q4Work(ctx, 55), cache, q, q_pos)
    _refused(pc.PC_ERR_CAPACITY, pc.pc_q4_attend, work, cache, q.expand(3, -1, -1).contiguous(), q_pos.expand(3, -1).contiguous())
    _refused(pc.PC_ERR_INVALID_ARG, pc.pc_q4_attend, work, cache, q[:0], q_pos[:0])
    with pytest.raises(AssertionError, match="contiguous"):
        pc.pc_q4_attend(work, cache, q.transpose(1, 2), q_pos)
    _refused(pc.PC_ERR_INVALID_ARG, pc.Q4Work, ctx, 0)
    assert pc.pc_poll_status(ctx) == pc.PC_OK


def test_positions_outside_the_rotary_table_are_recorded():
    c = Case("lumos", 16, 40, 1)
    c.q_pos[0, 1] = 400
    pc.pc_q4_attend(c.work, c.cache, c.q, c.q_pos)
    assert pc.pc_poll_status(c.ctx) == pc.PC_ERR_INVALID_ARG
    c.q_pos[0, 1] = 0
    c.q_pos[0, 0] = 599
    c.hist.t_shift = 1                                   # 600 is outside
    pc.pc_q4_attend(c.work, c.cache, c.q, c.q_pos)
    assert pc.pc_poll_status(c.ctx) == pc.PC_ERR_INVALID_ARG


@pytest.mark.parametrize("n_q,frames", [(1, False), (5, False), (40, True)])
def test_queries_that_are_not_finite_stay_so_and_alone(n_q, frames):
    c = Case("lumos", 96, 384, n_q, shift=8, frames=frames)
    clean = _np(pc.pc_q4_attend(c.work, c.cache, c.q, c.q_pos))
    c.q[n_q - 1, 2, 7] = float("nan")
    c.q[n_q // 2, 11, 90] = float("-inf")
    got = _np(pc.pc_q4_attend(c.work, c.cache, c.q, c.q_pos))
    off = np.zeros(got.shape[:2], bool)
    off[n_q - 1, 2] = off[n_q // 2, 11] = True
    assert np.isnan(got[off]).all()
    # the rows beside them may be scaled at another step: one rounding of the output and of the probabilities
    assert (np.abs(got - clean)[~off] <= 2.0 ** -7 * np.abs(clean[~off]) + 2.0 ** -9).all()
    pc.pc_poll_status(c.ctx)


def test_frame_queries_beyond_half_precision_are_recorded():
    c = Case("lumos", 96, 384, 40, frames=True)
    pc.pc_q4_attend(c.work, c.cache, c.q, c.q_pos)
    assert pc.pc_poll_status(c.ctx) == pc.PC_OK
    c.q[3, 5, 0] = 1e8
    out = pc.pc_q4_attend(c.work, c.cache, c.q, c.q_pos)
    assert pc.pc_poll_status(c.ctx) == pc.PC_ERR_INVALID_ARG
    assert torch.isfinite(out).all()
