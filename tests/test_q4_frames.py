"""Frames over the 4-bit cache where a CTA takes many key tiles, goes from one item to the next, and shares items with others: the form of the tensor-core
attention with keys and values in three places, in numbers of steps that its pipeline goes round in.

Keys of a tile share a direction (of the queries', by an amount of the tile's own) and values an offset, so that a tile taken for another, taken twice or left
out shows in every output.  Tolerances: a key is rounded to fp16, so each of 128 products of a logit is off by up to 2^-12 of itself, to either side; their sum
passes t |q o k|_2 2^-12 / sqrt(d) with probability 2 exp(-t^2 / 2), and t = 8 leaves 2e-5 for all logits of all cases together.  With fp32
sums (48 additions), delta = (8 * 2^-12 + 48 * 2^-23) max_j |q o k_j|_2 / sqrt(d).  Outputs: (2 delta + 2^-11 for the probability and the value) sum p |v|,
fp16's last places of small probabilities, and bf16's rounding."""
from __future__ import annotations

import ctypes as C

import numpy as np
import pytest
import torch

from paper_2601_04359_b200 import binding as pc
from tests import q4_reference as ref

from .host_runtime import Case as HostCase, _library, rt  # noqa: F401

TILE = 128
# query / KV heads, queries, anchors, history, fixed key ranges; what is launched behind k_q4_front, and its CTAs on 148 SMs
CASES = {
    "frame": ((24, 8), 1008, 1136, 8064, 0),             # runs of 47 steps over 96 items of 72 tiles: every run crosses items, two-part items merged in the kernel
    "short_frame": ((24, 8), 1008, 1136, 2100, 0),       # runs of 17, items in up to three parts
    "few_items": ((8, 8), 300, 0, 5000, 0),              # items cut into equal ranges of five tiles
    "one_range": ((24, 8), 1600, 70, 650, 0),            # more items than CTAs, no boundary between segments on a tile
    "two_fixed": ((24, 8), 135, 37, 2500, 2),            # two fixed ranges an item, merged by a kernel of their own
    "odd_tiles": ((40, 8), 600, 300, 1229, 0),           # an odd number of query tiles
    "two_heads": ((16, 2), 700, 5, 6000, 0),
    "one_tile": ((8, 8), 100, 0, 9000, 2),               # a single query tile an item, whose second copy is dropped
    "four_fixed": ((16, 8), 70, 100, 8300, 4),
}
MERGED, COMBINED = ["k_attend_tc"], ["k_attend_tc", "k_combine"]
DIVISION = {"frame": (MERGED, 144), "short_frame": (COMBINED, 148), "few_items": (COMBINED, 128), "one_range": (MERGED, 148), "two_fixed": (COMBINED, 48),
            "odd_tiles": (MERGED, 104), "two_heads": (COMBINED, 144), "one_tile": (COMBINED, 16), "four_fixed": (COMBINED, 32)}


class _Q4Segment(C.Structure):
    _fields_ = [("rows", C.c_void_p), ("pos", C.c_void_p), ("weight", C.c_void_p), ("n_tokens", C.c_int32), ("capacity", C.c_int32), ("t_shift", C.c_int32)]


class _Q4Cache(C.Structure):
    _fields_ = [("anchors", _Q4Segment), ("history", _Q4Segment)]


def _tiles(*n):
    return sum(-(-x // TILE) for x in n)


def _items(heads, n_q):
    return heads[1] * -(-(heads[0] // heads[1] * -(-n_q // TILE)) // 2)


@pytest.mark.parametrize("name", list(CASES))
def test_runs_are_long(rt, name):
    heads, n_q, n_a, n_h, splits = CASES[name]
    c = HostCase(rt, heads=heads + (128,), n=1, total=1, anchors=1, max_q=n_q, max_keys=n_a + n_h)
    room = torch.empty(1 << 12, dtype=torch.uint8)
    at = (room.data_ptr() + 255) // 256 * 256              # nothing is read: an address stands for all
    seg = lambda n: _Q4Segment(at, at, None, n, n, 0)      # noqa: E731
    cache, work = _Q4Cache(seg(n_a), seg(n_h)), C.c_void_p()
    assert rt.lib.pc_set_kv_splits(c.ctx.handle, splits) == pc.PC_OK
    assert rt.lib.pc_q4_create(c.ctx.handle, n_a + n_h, pc.PC_Q4_FRAMES, C.byref(work)) == pc.PC_OK
    rt.reset()
    rt.lib.pc_q4_attend.argtypes = [C.c_void_p] * 5 + [C.c_int32] + [C.c_void_p] * 4
    assert rt.lib.pc_q4_attend(work, C.byref(cache), None, at, at, n_q, at, None, None, None) == pc.PC_OK
    kernels = [line.split()[1] for line in rt.log() if line.startswith("launch")]
    ctas = rt.lib.rt_blocks(b"k_attend_tc")
    rt.lib.pc_q4_destroy(work)
    steps = _items(heads, n_q) * _tiles(n_a, n_h) / ctas
    assert (kernels[1:], ctas) == DIVISION[name]
    assert steps >= 4


class Layer:
    """Queries, and a cache of rows that differ from tile to tile, all at position zero; the history's keys have been rebased."""

    def __init__(self, heads, n_q, n_a, n_h, splits=0):
        hq, hkv = heads
        self.n_q, self.g = n_q, hq // hkv
        rng = np.random.default_rng(n_h + n_q)
        base = rng.standard_normal((hkv, 128))
        self.ctx = pc.Context(hq, hkv, 128, pc.PC_BF16, 10000.0, (64, 8, 8), self.n_q, n_a + n_h)
        pc.pc_set_kv_splits(self.ctx, splits)
        segs = []
        for n, shift in ((n_a, 0), (n_h, 24)):
            seg = pc.Q4Segment.empty(self.ctx, n, t_shift=shift)
            tile = np.arange(n) // TILE
            amount, side = rng.uniform(-2, 2, (_tiles(n), hkv)) / 128 ** 0.5, 8.0 * rng.choice([-1.0, 1.0], (_tiles(n), hkv, 128))
            k = amount[tile][:, :, None] * base + 0.7 * rng.standard_normal((n, hkv, 128))
            v = side[tile] + rng.standard_normal((n, hkv, 128))
            if n:
                k, v = (torch.from_numpy(x).cuda().bfloat16() for x in (k, v))
                pc.pc_q4_store(self.ctx, pc.Segment(k, v, torch.zeros(n, 4, dtype=torch.int32, device="cuda"), n), seg)
            segs.append(seg)
        self.cache = pc.Q4Cache(*segs)
        self.q = torch.from_numpy(np.repeat(base, self.g, 0) + 0.5 * rng.standard_normal((self.n_q, hq, 128))).cuda().bfloat16()
        self.q_pos = torch.zeros(self.n_q, 4, dtype=torch.int32, device="cuda")
        self.work = pc.Q4Work(self.ctx, n_a + n_h, frames=True)

    def attend64(self, valid=None):
        """out, lse, max |q o k|_2 / sqrt(d), sum p |v|, what the last places of small probabilities come to, and sqrt(sum (p (step code + |low|))^2);
        self.mass: the mean probability of every token of the history."""
        d = 128
        pos = np.zeros((self.n_q, 4), np.int32)
        k, v, q, spread_v = [], [], [], []
        for seg in (self.cache.anchors, self.cache.history):
            if seg.n_tokens:
                held = ref.decode(seg.rows.cpu().numpy(), d)
                a, b = (torch.from_numpy(ref.values(x)).cuda() for x in held)
                spread_v.append(torch.from_numpy(ref.spread(held[1])).cuda())
                k.append(a)
                v.append(b)
                q.append(torch.from_numpy(ref.turn(self.q.double().cpu().numpy(), pos, seg.t_shift)).cuda())
        hq = self.q.shape[1]
        out, mag, noise = (torch.empty(self.n_q, hq, d, dtype=torch.float64, device="cuda") for _ in range(3))
        lse, off, places = (torch.empty(self.n_q, hq, dtype=torch.float64, device="cuda") for _ in range(3))
        values, spread_v = torch.cat(v), torch.cat(spread_v)
        n_h = self.cache.history.n_tokens
        self.mass = torch.zeros(n_h, dtype=torch.float64, device="cuda")
        for h in range(hq):
            x = torch.cat([a[:, h] @ b[:, h // self.g].T for a, b in zip(q, k)], 1) / d ** 0.5
            if valid is not None:
                x[:, len(values) - n_h:].masked_fill_(valid[None] == 0, -torch.inf)
            spread = torch.cat([(a[:, h] ** 2) @ (b[:, h // self.g] ** 2).T for a, b in zip(q, k)], 1).amax(1).sqrt() / d ** 0.5
            lse[:, h] = torch.logsumexp(x, 1)
            p = torch.exp(x - lse[:, h, None])
            self.mass += p[:, len(values) - n_h:].sum(0) / (self.n_q * hq)
            w = values[:, h // self.g]
            out[:, h], mag[:, h] = p @ w, p @ w.abs()
            off[:, h] = spread
            noise[:, h] = ((p ** 2) @ (spread_v[:, h // self.g] ** 2)).sqrt()
            places[:, h] = 2.0 ** -32 * p.amax(1) * w.abs().sum(0).amax()
        return out, lse, off, mag, places, noise


@pytest.mark.gpu
@pytest.mark.parametrize("name", list(CASES))
def test_frames_of_many_steps(name):
    layer = Layer(*CASES[name])
    out, lse = pc.pc_q4_attend(layer.work, layer.cache, layer.q, layer.q_pos, want_lse=True)
    assert pc.pc_poll_status(layer.ctx) == pc.PC_OK
    want, want_lse, spread, mag, places, _ = layer.attend64()
    delta = (8 * 2.0 ** -12 + 48 * 2.0 ** -23) * spread
    off = (lse.double() - want_lse).abs()
    assert (off <= delta + 2.0 ** -20 * (1 + want_lse.abs())).all(), float((off / delta).max())
    off, tol = (out.double() - want).abs(), (2 * delta + 2.0 ** -11)[..., None] * mag + 2.0 ** -8 * want.abs() + places[..., None]
    assert (off <= tol).all(), float((off / tol).max())
    # the same bits from call to call, and where the second part of an item is left to the call's last CTA
    again, lse2 = torch.empty_like(out), torch.empty_like(lse)
    for leave in (False, True, True, False):
        pc.pc_test_leave_parts(layer.ctx, leave)
        again.zero_()
        lse2.zero_()
        pc.pc_q4_attend(layer.work, layer.cache, layer.q, layer.q_pos, out=again, lse=lse2)
        assert pc.pc_poll_status(layer.ctx) == pc.PC_OK
        assert torch.equal(again, out) and torch.equal(lse2, lse)


@pytest.mark.gpu
@pytest.mark.parametrize("n,n_q,masked,weigh", [(30_011, 1, 0.0, False), (30_011, 1, 0.2, True), (9_007, 5, 0.0, True), (9_007, 16, 0.2, False),
                                                (8_064, 1008, 0.3, False), (8_064, 1008, 0.0, True), (8_064, 1008, 0.05, True)])
def test_many_keys_without_the_tensor_core_form(n, n_q, masked, weigh):
    """Few queries, and whole frames with a mask or weights: the ring of units goes round many times, all keys in play.  Sums over codes and lows of a key are up to 34 |q o k|_2 (sqrt(128) for
    the sum of absolute values, 3 for step code + |low| of rows like these), of which 48 additions and the queries' parts round 48 * 2^-23 + 2^-21;
    probabilities and their products with steps are two roundings of 2^-11 each, independent from key to key: 8 of their standard deviations."""
    layer = Layer((24, 8), n_q, 1000, n)
    valid = (torch.rand(n, generator=torch.Generator().manual_seed(n_q)) >= masked).to(torch.uint8).cuda() if masked else None
    work = pc.Q4Work(layer.ctx, n + 1000, weigh=weigh)
    start = layer.cache.history.weight = torch.rand(n, device="cuda")
    start = start.clone()
    out, lse = pc.pc_q4_attend(work, layer.cache, layer.q, layer.q_pos, valid=valid, weigh=(0.5, 3.0) if weigh else None, want_lse=True)
    assert pc.pc_poll_status(layer.ctx) == pc.PC_OK
    want, want_lse, spread, mag, places, noise = layer.attend64(valid)
    delta = 34 * (48 * 2.0 ** -23 + 2.0 ** -21) * spread
    off = (lse.double() - want_lse).abs()
    assert (off <= delta + 2.0 ** -20 * (1 + want_lse.abs())).all(), float((off / delta).max())
    off, tol = (out.double() - want).abs(), 2 * delta[..., None] * mag + 8 * 2.0 ** -10 * noise + 2.0 ** -8 * want.abs() + places[..., None]
    assert (off <= tol).all(), float((off / tol).max())
    if weigh:                                              # a probability is off by a logit's and an lse's delta, and what exponentials and sums round
        off, mass = (layer.cache.history.weight.double() - 0.5 * start.double() - 3.0 * layer.mass).abs(), 3.0 * layer.mass
        assert (off <= (2 * delta.max() + 2.0 ** -17) * mass + 2.0 ** -22 * layer.cache.history.weight).all(), float((off / mass).max())
    else:
        assert torch.equal(layer.cache.history.weight, start)
