"""Attention over the 4-bit cache where probabilities and steps are small: values far below one, steps that differ by token and by group, and a key
that leaves the others little.

Tolerances of calls of few queries, bf16 contexts (logits as in test_q4_cache: delta <= (48 * 2^-23 + 2^-21) S).  A probability is rounded to fp16 as
2^8 p / p_max, then times its step as fp16 again: 2^-11 of each at most, and half of fp16's last place, 2^-25, where that is more.  The step is
scaled by a power of two f that brings the largest of its 32 channels to 32 at least (or by 2^15, if that is less), so the last places are 2^-33 of p_max a
key for the lows, and 2^-33 / f <= 2^-38 of the largest step (or 2^-48) for each of up to 15 codes."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from paper_2601_04359_b200 import binding as pc
from tests import q4_reference as ref
from tests.test_q4_cache import SHAPES, _ctx, _np, _t

pytestmark = pytest.mark.gpu


def _decoded(seg, d):
    return [tuple(torch.from_numpy(x).cuda() for x in q) for q in ref.decode(seg.rows[:seg.n_tokens].cpu().numpy(), d)]


def _values(q):
    c, step, low = q
    grouped = c.unflatten(-1, (-1, ref.GROUP)) * step[..., None]
    return (low[..., None] + grouped).flatten(-2), (low.abs()[..., None] + grouped).flatten(-2)


def _attend64(q, seg, valid=None):
    """Queries and keys at position zero.  Returns out, lse, S, the sums of p (step code + |low|), the largest p of every row, and per channel
    what half of a last place costs: sum (step code + |low|) of the visible keys, and 15 times their number times the largest step of the channel's group."""
    n_q, hq, d = q.shape
    kq, vq = _decoded(seg, d)
    hkv = kq[0].shape[1]
    g = hq // hkv
    if valid is not None:
        kq, vq = ([x[valid.bool()] for x in t] for t in (kq, vq))
    (k, sk), (v, sv) = _values(kq), _values(vq)
    q64 = q.double().view(n_q, hkv, g, d)
    x = torch.einsum("ihgd,jhd->hgij", q64, k) / d ** 0.5
    lse = torch.logsumexp(x, -1)
    p = torch.exp(x - lse[..., None])
    home = lambda t: t.permute(2, 0, 1, 3).reshape(n_q, hq, d)                                          # noqa: E731
    out, mag_v = (home(torch.einsum("hgij,jhd->hgid", p, t)) for t in (v, sv))
    back = lambda t: t.permute(2, 0, 1).reshape(n_q, hq)                                                # noqa: E731
    mag_l = back((torch.einsum("ihgd,jhd->hgij", q64.abs(), sk) / d ** 0.5).amax(-1))
    per_head = lambda t: t.repeat_interleave(g, 0)[None]                                                # noqa: E731
    top = vq[1].amax(0).repeat_interleave(ref.GROUP, -1)
    places = torch.maximum(2.0 ** -38 * top, torch.full_like(top, 2.0 ** -48)) * 15 * len(v) + 2.0 ** -33 * sv.sum(0)
    return out, back(lse), mag_l, mag_v, back(p.amax(-1)), per_head(places)


class Small:
    def __init__(self, shape, n, n_q, v, q=None, keys=None, max_q=0, masked=0.0, frames=False, seed=0):
        hq, hkv, d, dtype = SHAPES[shape]
        rng = np.random.default_rng(seed + n)
        self.dtype = dtype
        self.ctx = _ctx(shape, max_q or n_q, n)
        self.seg = pc.Q4Segment.empty(self.ctx, n)
        k = rng.standard_normal((n, hkv, d)) if keys is None else keys
        pos = torch.zeros(n, 4, dtype=torch.int32, device="cuda")
        pc.pc_q4_store(self.ctx, pc.Segment(_t(k, dtype), _t(v, dtype), pos, n), self.seg)
        self.q = _t(rng.standard_normal((n_q, hq, d)) * 2.5 if q is None else q, dtype)
        self.q_pos = torch.zeros(n_q, 4, dtype=torch.int32, device="cuda")
        self.valid = torch.from_numpy((rng.random(n) >= masked).astype(np.uint8)).cuda() if masked else None
        self.work = pc.Q4Work(self.ctx, n, frames=frames)

    def run(self):
        cache = pc.Q4Cache(pc.Q4Segment.empty(self.ctx, 0), self.seg)
        out, lse = pc.pc_q4_attend(self.work, cache, self.q, self.q_pos, valid=self.valid, want_lse=True)
        assert pc.pc_poll_status(self.ctx) == pc.PC_OK
        return out.double(), lse.double()

    def check(self):
        out, lse = self.run()
        want, want_lse, mag_l, mag_v, p_max, places = _attend64(self.q, self.seg, self.valid)
        delta = (48 * 2.0 ** -23 + 2.0 ** -21) * mag_l
        p_off = 2 * delta + 2.0 ** -18
        f32 = self.dtype == "f32"
        tol = (p_off + (2.0 ** -20 if f32 else 2.0 ** -10))[..., None] * mag_v + (2.0 ** -23 if f32 else 2.0 ** -8) * want.abs()
        if not f32:
            tol = tol + p_max[..., None] * places
        off = (out - want).abs()
        assert torch.isfinite(out).all()
        assert (off <= tol).all(), float((off / tol.clamp_min(1e-300)).max())
        assert ((lse - want_lse).abs() <= delta + 2.0 ** -20 * (1 + want_lse.abs())).all()


CALLS = {"token": ("lumos", 30_000, 1, 0, 0.0), "token64": ("small", 9_000, 2, 0, 0.0), "few": ("one", 20_000, 3, 0, 0.3),
         "many_masked": ("lumos", 5_000, 300, 1008, 0.3)}


@pytest.mark.parametrize("call", list(CALLS))
@pytest.mark.parametrize("scale", [1.0, 1e-2, 1e-3, 1e-4])
def test_values_far_below_one(call, scale):
    shape, n, n_q, max_q, masked = CALLS[call]
    _, hkv, d, _ = SHAPES[shape]
    Small(shape, n, n_q, scale * np.random.default_rng(1).standard_normal((n, hkv, d)), max_q=max_q, masked=masked).check()


@pytest.mark.parametrize("call", ["token", "token64", "few", "many_masked"])
@pytest.mark.parametrize("kind", ["growing", "shrinking", "one_large", "groups"])
def test_steps_that_differ(call, kind):
    """Steps over a factor of 4,096: along the tokens, of one token in the middle, and from one group of channels to the next."""
    shape, n, n_q, max_q, masked = CALLS[call]
    _, hkv, d, _ = SHAPES[shape]
    v = np.random.default_rng(2).standard_normal((n, hkv, d)) * 1e-3
    ramp = 2.0 ** (12 * np.arange(n) / n)
    if kind == "growing":
        v *= ramp[:, None, None]
    elif kind == "shrinking":
        v *= ramp[::-1, None, None]
    elif kind == "one_large":
        v[n // 2 + 5] *= 4096
    else:
        v *= 2.0 ** (4 * (np.arange(d) // 32))
    Small(shape, n, n_q, v, max_q=max_q, masked=masked).check()


def _dominant(shape, n, n_q, c, scale, silent, others=1.0, **kw):
    """All queries of a KV head alike, one key c times that query (about 11.3 c above the others' mean); silent: its value is zero, the others' are
    around 4 * scale, so that the output is what the others still get."""
    hq, hkv, d, _ = SHAPES[shape]
    rng = np.random.default_rng(3)
    base = rng.standard_normal((hkv, d))
    base *= (d ** 0.5 / np.sqrt((base ** 2).sum(-1)))[:, None]
    k = others * rng.standard_normal((n, hkv, d))
    v = scale * (4.0 * silent + rng.standard_normal((n, hkv, d)))
    at = 7
    k[at] = c * base
    if silent:
        v[at] = 0.0
    q = np.broadcast_to(np.repeat(base, hq // hkv, 0), (n_q, hq, d))
    return Small(shape, n, n_q, v, q=q, keys=k, **kw)


@pytest.mark.parametrize("shape,n,n_q,max_q", [("lumos", 20_000, 1, 0), ("lumos", 5_000, 200, 1008), ("small", 6_000, 2, 0), ("lumos_f32", 4_000, 2, 0)])
@pytest.mark.parametrize("c", [0.9, 1.2, 1.7])
@pytest.mark.parametrize("scale,silent", [(1.0, False), (1e-2, False), (1e-3, False), (1.0, True), (1e-2, True)])
def test_a_key_that_leaves_the_others_little(shape, n, n_q, max_q, c, scale, silent):
    if SHAPES[shape][2] == 64:
        c *= 2 ** 0.5
    _dominant(shape, n, n_q, c, scale, silent, max_q=max_q).check()


@pytest.mark.parametrize("c", [1.7, 2.2, 2.4])
def test_a_key_that_leaves_the_others_little_fp32(c):
    """fp32 contexts have no last places to reckon with: down to 2^-39 of the largest probability and beyond."""
    _dominant("lumos_f32", 4_000, 2, c, 1.0, True, others=0.05).check()


@pytest.mark.parametrize("n,n_q", [(3_000, 40), (300, 130)])
@pytest.mark.parametrize("c,scale", [(1.2, 1.0), (1.55, 1.0), (1.7, 1.0), (1.7, 1e-2)])
def test_a_key_that_leaves_the_others_little_in_a_frame(n, n_q, c, scale):
    """Tolerances as in test_frames_on_the_tensor_core_kernel, and half of fp16's last place of a probability, 2^-25, which is held as 2^7 p / p_max at least."""
    case = _dominant("lumos", n, n_q, c, scale, True, others=0.05, frames=True)
    out, lse = case.run()
    want, want_lse, mag_l, mag_v, p_max, _ = _attend64(case.q, case.seg)
    delta = (2.0 ** -12 + 48 * 2.0 ** -23) * mag_l
    assert ((lse - want_lse).abs() <= delta + 2.0 ** -20 * (1 + want_lse.abs())).all()
    sv = _values(_decoded(case.seg, 128)[1])[1].sum(0).repeat_interleave(3, 0)[None]                  # of the query heads' KV heads
    tol = (2 * delta + 2.0 ** -11)[..., None] * mag_v + 2.0 ** -8 * want.abs() + 2.0 ** -32 * p_max[..., None] * sv
    assert ((out - want).abs() <= tol).all(), float(((out - want).abs() / tol).max())


@pytest.mark.parametrize("shape,n_q", [("lumos", 1), ("lumos", 5), ("tiny_f32", 1), ("tiny_f32", 3)])
def test_queries_up_to_the_largest(shape, n_q):
    """Queries that rotation and log2(e) / sqrt(d) leave below 2^109 are taken as they are; beyond it they are scaled down, and that is recorded."""
    hq, hkv, d, _ = SHAPES[shape]
    rng = np.random.default_rng(9)
    q = rng.standard_normal((n_q, hq, d))
    case = Small(shape, 100, n_q, rng.standard_normal((100, hkv, d)), q=q)
    clean, clean_lse = case.run()
    case.q[0, 1] *= 1e31                                  # 2^103 and less
    _, lse = case.run()
    _, want, mag_l, _, _, _ = _attend64(case.q, case.seg)
    assert ((lse - want).abs() <= (48 * 2.0 ** -23 + 2.0 ** -21) * mag_l + 2.0 ** -20 * (1 + want.abs())).all()
    case.q[0, 1, :] = 0.0
    case.q[0, 1, 5] = 3e38
    cache = pc.Q4Cache(pc.Q4Segment.empty(case.ctx, 0), case.seg)
    out, lse = pc.pc_q4_attend(case.work, cache, case.q, case.q_pos, want_lse=True)
    assert pc.pc_poll_status(case.ctx) == pc.PC_ERR_INVALID_ARG
    assert torch.isfinite(out).all() and torch.isfinite(lse).all() and lse[0, 1] > 1e31
    others = torch.ones(n_q, hq, dtype=torch.bool, device="cuda")
    others[0, 1] = False
    assert ((lse.double() - clean_lse).abs()[others] <= 1e-5).all()
    case.q[0, 1] = 3e38                                   # sums over channels as well
    out, lse = pc.pc_q4_attend(case.work, cache, case.q, case.q_pos, want_lse=True)
    assert pc.pc_poll_status(case.ctx) == pc.PC_ERR_INVALID_ARG
    assert torch.isfinite(out).all() and torch.isfinite(lse).all()
