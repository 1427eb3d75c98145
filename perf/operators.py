"""Timed cases of the 4-bit cache: rows written and read back, attention of single tokens, of a few and of a whole frame over
it, attention weights accumulated on the way, and eviction of the tokens that received the least.

A case is a dict of plain values.  ``op`` names the operator; the rest are sizes: query / KV heads and head dimension,
storage type, tokens of the anchors and of the history, query tokens, and what an eviction keeps.  Inputs are what a video
generator's layer brings: unit-variance Q, K and V, for bf16 with a +-4 bias on 2 % of the K and V channels, and
(t, h, w) coordinates scaled by (4, 8, 8).

Formulas.  A group of 32 channels x of a row is held as low = fp16(min x), step = fp16((max x - low) / 15) and codes
c = clamp(rint((x - low) / step), 0, 15), and stands for low + step c.  Keys are held rotated, at (t + t_shift, h, w).
Attention: out = softmax(R q . k / sqrt(d)) v over anchors ++ unmasked history; weight <- decay weight + gain mean p."""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

BASE = 10000.0
GROUP = 32
DECAY, GAIN = 0.98, 1.0
F15 = float(np.float32(1.0) / np.float32(15.0))


def _case(name, op, n_hist, *, heads=(24, 8, 128), dtype="bf16", n_anchor=0, n_q=1, shift=0, masked=0.0, weigh=False, keep=0, recent=0,
          delta_t=0, bits=4):
    c = {"op": op, "q_heads": heads[0], "kv_heads": heads[1], "head_dim": heads[2], "dtype": dtype, "n_anchor": n_anchor,
         "n_hist": n_hist, "n_q": n_q, "shift": shift, "masked": masked, "weigh": weigh, "keep": keep, "recent": recent,
         "delta_t": delta_t, "bits": bits}
    return dict(c, name=name) if name else c


def listed():
    tiny = (4, 2, 64)
    return [
        # one 64-token fp32 frame of the smallest configuration, written and read back: launches and latency
        _case("store_tiny_f32", "store", 64, heads=tiny, dtype="f32"),
        # the frame that was just generated enters the cache (and is read back for a call that wants 16 bits)
        _case("store_frame", "store", 1008),
        # a whole history is moved into four bits at once, an odd count of tokens
        _case("store_24_frames", "store", 24 * 1008 + 1),
        # a single text token over the smallest fp32 cache
        _case("token_tiny_f32", "attend", 384, heads=tiny, dtype="f32", n_anchor=96),
        # a single token early in a generation: anchors and 12 frames, the history rebased by two frames since it was written
        _case("token_12_frames", "attend", 12 * 1008, n_anchor=1136, shift=8),
        # a single token at the end of a 48-frame generation
        _case("token_47_frames", "attend", 47 * 1008, n_anchor=1136),
        # the same with the weights that a later eviction goes by
        _case("token_weigh_24_frames", "attend", 24 * 1008, n_anchor=1136, weigh=True),
        # five tokens at once, ragged lengths, a cache mask, 32 / 8 heads, weights
        _case("few_masked_weigh", "attend", 4999, heads=(32, 8, 128), n_anchor=37, n_q=5, masked=0.1, weigh=True, shift=4),
        # a whole frame of queries over a compacted cache
        _case("frame_packed_cache", "attend", 8064, n_anchor=1136, n_q=1008),
        # a small clip's 16-bit history cut to 300 tokens, the newest frame kept
        _case("evict_small_16bit", "evict", 675, keep=300, recent=135, bits=16),
        # a 24-frame history in 16 bits cut to a quarter, one frame dropped from the time axis
        _case("evict_24_frames_16bit", "evict", 24 * 1008, keep=6048, recent=1008, delta_t=4, bits=16),
        # a 47-frame history in four bits cut to two whole frames and 6048 heavy hitters, read back
        _case("evict_47_frames", "evict", 47 * 1008, keep=8064, recent=2016, delta_t=4),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    small = rng.random() < 0.15
    heads = (4, 2, 64) if small else rng.choice([(24, 8, 128), (24, 8, 128), (32, 8, 128), (16, 4, 128), (8, 8, 128), (24, 12, 128)])
    dtype = "f32" if small else "bf16"
    op = rng.choice(["store", "attend", "attend", "attend", "evict"])
    most = 4000 if small else 48000 * 8 // max(8, heads[1])
    if op == "store":
        return _case("", op, _log_int(rng, 1, most // 2), heads=heads, dtype=dtype)
    if op == "evict":
        n = _log_int(rng, 16, most)
        keep = max(1, int(n * rng.uniform(0.1, 0.8)))
        return _case("", op, n, heads=heads, dtype=dtype, keep=keep, recent=int(keep * rng.choice([0.0, 0.1, 0.3])),
                     delta_t=rng.choice([0, 4]), bits=rng.choice([4, 16]))
    n = _log_int(rng, 16, most)
    n_anchor = _log_int(rng, 1, 1200)
    kind = rng.choice(["token", "token", "few", "frame"])
    n_q = 1 if kind == "token" else _log_int(rng, 2, 24) if kind == "few" else _log_int(rng, 64, 64 if small else 1008)
    weigh = kind != "frame" and rng.random() < 0.4
    masked = rng.choice([0.0, 0.05, 0.3]) if kind != "frame" else 0.0
    if kind == "frame":
        n = min(n, 9000)
    return _case("", op, n, heads=heads, dtype=dtype, n_anchor=n_anchor, n_q=n_q, shift=rng.choice([0, 4, 24]), masked=masked, weigh=weigh)


# ---------------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------------
def _axes(d):
    """axis (0, 1, 2) and frequency of each rotary pair"""
    i = np.arange(d // 2)
    axis = i % 3
    n_axis = np.array([(axis == a).sum() for a in range(3)])
    return axis, BASE ** (-(i // 3) / n_axis[axis])


def _max_pos(c):
    frames = -(-(c["n_hist"] + c["n_q"]) // 1008) + 1
    return (max(1300, 128 + 4 * (frames + 3)), 1300, 1300)


def _table(c, extra):
    """[3][positions][pairs] (cos, sin) of position x frequency, zero where a pair turns with another axis"""
    d = c["head_dim"]
    axis, freq = _axes(d)
    n = max(_max_pos(c)) + extra
    ang = np.arange(n, dtype=np.float64)[:, None] * freq
    t = np.stack([np.cos(ang), np.sin(ang)], -1).astype(np.float32)
    return torch.from_numpy(t).cuda(), torch.from_numpy(axis).cuda()


class _State:
    pass


def _positions(n, first):
    """(t, h, w, tag) of n consecutive tokens of frames of 24 x 42, from frame `first` on"""
    i = torch.arange(n, device="cuda", dtype=torch.int32)
    f, r = i // 1008, i % 1008
    return torch.stack([128 + 4 * (first + f), 8 * (r // 42), 8 * (r % 42), i], 1).contiguous()


def _dtype(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _raw(c, gen, n, bias):
    shape = (n, c["kv_heads"], c["head_dim"])
    x = torch.randn(shape, generator=gen, device="cuda")
    return (x + bias if bias is not None else x).to(_dtype(c)).contiguous()


def _inputs(c, seed):
    """The tensors of a case from the seed alone."""
    s = _State()
    gen = torch.Generator(device="cuda").manual_seed(int(seed) % (1 << 62))
    slots = c["kv_heads"] * c["head_dim"]
    bias = [None, None]
    if c["dtype"] == "bf16":
        for i in range(2):
            b = torch.zeros(slots, device="cuda")
            at = torch.randperm(slots, generator=gen, device="cuda")[: max(1, slots // 50)]
            b[at] = 4.0 * (1 - 2 * torch.randint(0, 2, at.shape, generator=gen, device="cuda").float())
            bias[i] = b.view(c["kv_heads"], c["head_dim"])
    s.hist = (_raw(c, gen, c["n_hist"], bias[0]), _raw(c, gen, c["n_hist"], bias[1]), _positions(c["n_hist"], 1))
    if c["op"] == "attend":
        n = c["n_anchor"]
        i = torch.arange(n, device="cuda", dtype=torch.int32)
        s.anchor = (_raw(c, gen, n, bias[0]), _raw(c, gen, n, bias[1]), torch.stack([i, i, i, i], 1).contiguous())
        s.q = torch.randn(c["n_q"], c["q_heads"], c["head_dim"], generator=gen, device="cuda").to(_dtype(c))
        s.q_pos = _positions(c["n_q"], 1 + -(-c["n_hist"] // 1008))
        s.valid = (torch.rand(c["n_hist"], generator=gen, device="cuda") >= c["masked"]).to(torch.uint8) if c["masked"] else None
    # what tokens have received so far: heavy-tailed, with tokens that nothing has looked at yet
    w = torch.randn(c["n_hist"], generator=gen, device="cuda").exp() / c["n_hist"]
    w[torch.rand(c["n_hist"], generator=gen, device="cuda") < 0.02] = 0.0
    s.weight = w
    return s


def prepare(case, seed):
    """Inputs, and what a program keeps beside them: the cache that the rows were written to, output buffers, workspaces."""
    c = dict(case)
    s = _inputs(c, seed)
    s.c, s.own = c, own
    if not own:
        s.tab = _table(c, c["shift"])
        if c["op"] == "attend":
            s.anchor_q4 = _quantise_rows(s.tab, *s.anchor, 0)
            s.hist_q4 = _quantise_rows(s.tab, *s.hist, c["shift"])
        if c["op"] == "evict" and c["bits"] == 4:
            s.hist_q4 = _quantise_rows(s.tab, *s.hist, 0)
        return s
    from paper_2601_04359_b200 import binding as pc
    n, hkv, d = c["n_hist"], c["kv_heads"], c["head_dim"]
    dt = pc.PC_BF16 if c["dtype"] == "bf16" else pc.PC_F32
    s.ctx = pc.Context(c["q_heads"], hkv, d, dt, BASE, _max_pos(c), max(1, c["n_q"]), c["n_anchor"] + n)
    s.raw = pc.Segment(*s.hist, n)
    if c["op"] == "store":
        s.seg = pc.Q4Segment.empty(s.ctx, n)
        s.back = pc.Segment(torch.empty_like(s.hist[0]), torch.empty_like(s.hist[1]), torch.empty_like(s.hist[2]), 0)
    elif c["op"] == "attend":
        hist = pc.Q4Segment.empty(s.ctx, n, t_shift=c["shift"], weight=c["weigh"])
        anchors = pc.Q4Segment.empty(s.ctx, c["n_anchor"])
        pc.pc_q4_store(s.ctx, s.raw, hist, 0)
        pc.pc_q4_store(s.ctx, pc.Segment(*s.anchor, c["n_anchor"]), anchors, 0)
        if c["weigh"]:
            hist.weight.copy_(s.weight)
        s.cache = pc.Q4Cache(anchors, hist)
        s.work = pc.Q4Work(s.ctx, c["n_anchor"] + n, frames=c["n_q"] > 16, weigh=c["weigh"])
        s.out = torch.empty_like(s.q)
        s.lse = torch.empty(c["n_q"], c["q_heads"], device="cuda")
    else:
        s.sel = torch.empty(c["keep"], dtype=torch.int32, device="cuda")
        if c["bits"] == 4:
            s.seg = pc.Q4Segment.empty(s.ctx, n, weight=True)
            pc.pc_q4_store(s.ctx, s.raw, s.seg, 0)
            s.seg.weight.copy_(s.weight)
            s.dst = pc.Q4Segment.empty(s.ctx, c["keep"], weight=True)
        else:
            s.dst_weight = torch.empty(c["keep"], device="cuda")
        s.back = pc.Segment(s.hist[0].new_empty((c["keep"], hkv, d)), s.hist[1].new_empty((c["keep"], hkv, d)),
                            s.hist[2].new_empty((c["keep"], 4)), 0)
    return s


# ---------------------------------------------------------------------------------------------------------------------
# the plain form
# ---------------------------------------------------------------------------------------------------------------------
def _cos_sin(tab, pos, shift):
    t, axis = tab
    p = pos[:, :3].long()
    p = torch.stack([p[:, 0] + shift, p[:, 1], p[:, 2]], 1)[:, axis]             # [n][pairs]
    cs = t[p, torch.arange(len(axis), device=p.device)]
    return cs[..., 0][:, None, :], cs[..., 1][:, None, :]


def _rotate(tab, x, pos, shift, back=False):
    c, s = _cos_sin(tab, pos, shift)
    if back:
        s = -s
    x0, x1 = x[..., 0::2], x[..., 1::2]
    return torch.stack([x0 * c - x1 * s, x0 * s + x1 * c], -1).flatten(-2)


def _quantise(x):
    """Rows in fp32 -> codes (two to a byte), steps and lows"""
    g = x.view(*x.shape[:-1], -1, GROUP)
    lo = g.amin(-1).clamp(-65504.0, 65504.0).half()
    step = ((g.amax(-1).clamp(-65504.0, 65504.0) - lo.float()) * F15).half()
    inv = torch.where(step > 0, 1.0 / step.float(), torch.zeros((), device=x.device))
    code = torch.round((g - lo.float()[..., None]) * inv[..., None]).clamp(0.0, 15.0).to(torch.uint8).flatten(-2)
    return code[..., 0::2] | (code[..., 1::2] << 4), step, lo


def _values(q):
    """What the codes stand for, in fp32"""
    byte, step, lo = q
    code = torch.stack([byte & 15, byte >> 4], -1).flatten(-2).float()
    g = code.view(*code.shape[:-1], -1, GROUP)
    return (lo.float()[..., None] + step.float()[..., None] * g).flatten(-2)


def _quantise_rows(tab, k, v, pos, shift):
    return _quantise(_rotate(tab, k.float(), pos, shift)), _quantise(v.float())


def _attend(s):
    c = s.c
    n_q, hq, hkv, d = c["n_q"], c["q_heads"], c["kv_heads"], c["head_dim"]
    logits, values = [], []
    for (k4, v4), shift in ((s.anchor_q4, 0), (s.hist_q4, c["shift"])):
        q = _rotate(s.tab, s.q.float(), s.q_pos, shift).view(n_q, hkv, hq // hkv, d).permute(1, 2, 0, 3).reshape(hkv, -1, d)
        logits.append(torch.matmul(q, _values(k4).permute(1, 2, 0)) * (1.0 / math.sqrt(d)))
        values.append(_values(v4).permute(1, 0, 2))
    if s.valid is not None:
        logits[1] = torch.where(s.valid.bool(), logits[1], torch.full((), -math.inf, device="cuda"))
    x = torch.cat(logits, -1)                                                     # [Hkv][G n_q][keys]
    m = x.amax(-1, keepdim=True)
    e = torch.exp(x - m)
    l = e.sum(-1, keepdim=True)
    p = e / l
    out = torch.matmul(p, torch.cat(values, 1))
    home = lambda y: y.view(hkv, hq // hkv, n_q, -1).permute(2, 0, 1, 3).reshape(n_q, hq, -1)     # noqa: E731
    got = {"out": home(out).to(s.q.dtype), "lse": home(m + torch.log(l))[..., 0]}
    if c["weigh"]:
        s.weight.mul_(DECAY).add_(p[..., c["n_anchor"]:].sum((0, 1)) * (GAIN / (n_q * hq)))
        got["weight"] = s.weight
    return got


def _evict(s):
    c = s.c
    older = c["n_hist"] - c["recent"]
    order = torch.sort(s.weight[:older], descending=True, stable=True).indices[: c["keep"] - c["recent"]]
    sel = torch.cat([torch.sort(order).values, torch.arange(older, c["n_hist"], device="cuda")])
    pos = s.hist[2][sel] - torch.tensor([c["delta_t"], 0, 0, 0], dtype=torch.int32, device="cuda")
    if c["bits"] == 16:
        k, v = s.hist[0][sel], s.hist[1][sel]
    else:
        k, v = ([x[sel] for x in q] for q in s.hist_q4)
        k, v = _rotate(s.tab, _values(k), pos, c["delta_t"], back=True).to(_dtype(c)), _values(v).to(_dtype(c))
    return {"sel": sel.int(), "k": k, "v": v, "pos": pos, "weight": s.weight[sel]}


def _plain(s):
    c = s.c
    if c["op"] == "attend":
        return _attend(s)
    if c["op"] == "evict":
        return _evict(s)
    k4, v4 = _quantise_rows(s.tab, *s.hist, 0)
    return {"k": _rotate(s.tab, _values(k4), s.hist[2], 0, back=True).to(_dtype(c)), "v": _values(v4).to(_dtype(c)), "pos": s.hist[2].clone()}


# ---------------------------------------------------------------------------------------------------------------------
# the calls that a user makes
# ---------------------------------------------------------------------------------------------------------------------
def _library(s):
    from paper_2601_04359_b200 import binding as pc
    c = s.c
    if c["op"] == "attend":
        pc.pc_q4_attend(s.work, s.cache, s.q, s.q_pos, valid=s.valid, weigh=(DECAY, GAIN) if c["weigh"] else None, out=s.out, lse=s.lse)
        got = {"out": s.out, "lse": s.lse}
        if c["weigh"]:
            got["weight"] = s.cache.history.weight
        return got
    if c["op"] == "store":
        pc.pc_q4_store(s.ctx, s.raw, s.seg, 0)
        pc.pc_q4_load(s.ctx, s.seg, 0, c["n_hist"], s.back)
        return {"k": s.back.k, "v": s.back.v, "pos": s.back.pos}
    if c["bits"] == 4:
        pc.pc_q4_evict(s.ctx, s.seg, c["keep"], c["recent"], s.dst, delta_t=c["delta_t"], sel_idx=s.sel)
        pc.pc_q4_load(s.ctx, s.dst, 0, c["keep"], s.back)
        return {"sel": s.sel, "k": s.back.k, "v": s.back.v, "pos": s.dst.pos, "weight": s.dst.weight}
    pc.pc_evict(s.ctx, s.raw, s.weight, c["keep"], c["recent"], s.back, s.dst_weight, delta_t=c["delta_t"], sel_idx=s.sel)
    return {"sel": s.sel, "k": s.back.k, "v": s.back.v, "pos": s.back.pos, "weight": s.dst_weight}


def run(state):
    return _library(state) if state.own else _plain(state)


# ---------------------------------------------------------------------------------------------------------------------
# work, and the definition in 64 bits
# ---------------------------------------------------------------------------------------------------------------------
def work(case):
    c = case
    hkv, d, n = c["kv_heads"], c["head_dim"], c["n_hist"]
    elem = 2 if c["dtype"] == "bf16" else 4
    raw, held = 2 * hkv * d * elem, 2 * hkv * d * 5 // 8               # bytes of a token's keys and values, 16 or 32 bits and four
    if c["op"] == "store":
        return {"bytes": n * (2 * raw + 2 * held + 4 * 16 + 4), "flops": n * 2 * hkv * d * 8}
    if c["op"] == "evict":
        row = raw if c["bits"] == 16 else held
        back = 0 if c["bits"] == 16 else c["keep"] * (held + raw)
        return {"bytes": 4 * n + c["keep"] * (2 * (row + 20) + 4) + back, "flops": n}
    keys = n + c["n_anchor"]
    b = keys * held + c["n_q"] * c["q_heads"] * (2 * d * elem + 4) + (8 * n if c["weigh"] else 0) + (n if c["masked"] else 0)
    return {"bytes": b, "flops": 4 * c["n_q"] * c["q_heads"] * d * keys}


def _turn(c, x, pos, shift, sign=1.0):
    """The rotary embedding as a product of complex numbers"""
    axis, freq = _axes(c["head_dim"])
    a = torch.from_numpy(axis).cuda()
    p = pos[:, :3].double()
    p[:, 0] += shift
    ang = p[:, a] * torch.from_numpy(freq).cuda()
    z = torch.view_as_complex(x.double().reshape(*x.shape[:-1], -1, 2).contiguous())
    return torch.view_as_real(z * torch.polar(torch.ones_like(ang), sign * ang)[:, None, :]).flatten(-2)


def _held(x):
    """What four bits keep of rows in 64 bits"""
    g = x.unflatten(-1, (-1, GROUP))
    lo = g.min(-1, keepdim=True).values.half().double()
    step = ((g.max(-1, keepdim=True).values - lo) / 15.0).half().double()
    code = torch.where(step > 0, (g - lo) / step, torch.zeros_like(g)).round().clamp(0, 15)
    return (lo + step * code).flatten(-2)


def exact(case, seed):
    c = dict(case)
    s = _inputs(c, seed)
    if c["op"] == "store":
        k = _turn(c, _held(_turn(c, s.hist[0], s.hist[2], 0)), s.hist[2], 0, -1.0)
        return {"k": k, "v": _held(s.hist[1].double()), "pos": s.hist[2]}
    if c["op"] == "evict":
        older = c["n_hist"] - c["recent"]
        w = s.weight.cpu().numpy()
        best = np.lexsort((np.arange(older), -w[:older].astype(np.float64)))[: c["keep"] - c["recent"]]
        sel = torch.from_numpy(np.concatenate([np.sort(best), np.arange(older, c["n_hist"])])).cuda()
        k, v, pos = (x[sel] for x in s.hist)
        if c["bits"] == 4:
            k = _turn(c, _held(_turn(c, k, pos, 0)), pos, 0, -1.0)
            v = _held(v.double())
        pos = pos.clone()
        pos[:, 0] -= c["delta_t"]
        return {"sel": sel.int(), "k": k.double(), "v": v.double(), "pos": pos, "weight": s.weight[sel].double()}
    n_q, hq, hkv = c["n_q"], c["q_heads"], c["kv_heads"]
    out = torch.empty(n_q, hq, c["head_dim"], dtype=torch.float64, device="cuda")
    lse = torch.empty(n_q, hq, dtype=torch.float64, device="cuda")
    mass = torch.zeros(c["n_hist"], dtype=torch.float64, device="cuda")
    parts = [(s.anchor, 0), (s.hist, c["shift"])]
    ks = [_held(_turn(c, p[0], p[2], sh)) for p, sh in parts]
    v = torch.cat([_held(p[1].double()) for p, _ in parts])
    qs = [_turn(c, s.q, s.q_pos, sh) for _, sh in parts]
    for h in range(hq):
        g = h * hkv // hq
        x = torch.cat([q[:, h] @ k[:, g].T for q, k in zip(qs, ks)], 1) / math.sqrt(c["head_dim"])
        if s.valid is not None:
            x[:, c["n_anchor"]:].masked_fill_(s.valid[None] == 0, -math.inf)
        lse[:, h] = torch.logsumexp(x, 1)
        p = torch.exp(x - lse[:, h, None])
        out[:, h] = p @ v[:, g]
        mass += p[:, c["n_anchor"]:].sum(0)
    got = {"out": out, "lse": lse}
    if c["weigh"]:
        got["weight"] = DECAY * s.weight.double() + GAIN / (n_q * hq) * mass
    return got
