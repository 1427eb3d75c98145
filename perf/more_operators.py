"""Timed cases of the paged cache: keys and values appended with their rotation, attention of whole prompts (causal, packed, ragged) and
of frames, and attention of single tokens or a few of a batch whose sequences share a long prefix.

A case is a dict of plain values.  ``op`` is "append" or "attend"; the rest are sizes: query / KV heads and head dimension, storage type,
tokens of a page, sequences, tokens of the prefix they share, the range of the tokens that a sequence holds of its own before the
call, the range of the rows that it brings, and whether attention is causal.  Lengths are spread over their ranges by the case
alone.  Inputs are what the layers of a video generator bring: unit-variance Q, K and V, for bf16 with a +-4 bias on 2 % of the K and V
channels, (t, h, w) coordinates scaled by (4, 8, 8), and pages in the order in which a pool gives them out, which is none.

Formulas.  Keys are held rotated at their (t, h, w): pair i of a head turns with axis i mod 3.  Row i of the n rows of a sequence with L tokens of its own (the
rows' own tokens included) sees the whole prefix and, of its own tokens, those up to L - n + i (all of them where attention is not causal):
out = softmax(R q . k / sqrt(d)) v."""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

BASE = 10000.0
MAX_POS = (1300, 1300, 1300)
TEXT, ROWS, COLS = 128, 24, 42                 # a prompt's text, and the latent grid of a frame
FRAME = ROWS * COLS


def _case(name, op, seqs, *, heads=(24, 8, 128), dtype="bf16", page=64, prefix=0, before=(0, 0), rows=(1, 1), causal=True):
    c = {"op": op, "q_heads": heads[0], "kv_heads": heads[1], "head_dim": heads[2], "dtype": dtype, "page": page, "seqs": seqs, "prefix": prefix,
         "before_lo": before[0], "before_hi": before[1], "rows_lo": rows[0], "rows_hi": rows[1], "causal": causal}
    return dict(c, name=name) if name else c


def listed():
    tiny = (4, 2, 64)
    return [
        # every sample of a prompt has generated one token: launches and latency
        _case("append_token_8", "append", 8, page=16, before=(0, 300)),
        # eight samples have finished a frame each
        _case("append_8_frames", "append", 8, before=(0, 2016), rows=(FRAME, FRAME)),
        # prompts of all lengths enter the cache at once
        _case("append_prompts", "append", 40, heads=(32, 8, 128), page=32, rows=(1, 1136)),
        # two short prompts of the smallest fp32 configuration
        _case("prompts_tiny_f32", "attend", 2, heads=tiny, dtype="f32", page=16, rows=(37, 96)),
        # one prompt of text and a conditioning image
        _case("prompt_text_image", "attend", 1, rows=(TEXT + FRAME, TEXT + FRAME)),
        # prompts of all lengths packed into one call
        _case("prompts_packed", "attend", 12, heads=(32, 8, 128), page=32, rows=(17, 1136)),
        # a long prompt, text and eight frames and one token more
        _case("prompt_8193", "attend", 1, page=128, rows=(TEXT + 8 * FRAME + 1, TEXT + 8 * FRAME + 1)),
        # the next frame of four samples over their shared prompt and the frames that each has so far
        _case("frame_of_4_samples", "attend", 4, prefix=TEXT + FRAME, before=(2 * FRAME, 2 * FRAME), rows=(FRAME, FRAME), causal=False),
        # a token of each of four samples early on
        _case("token_4_samples", "attend", 4, prefix=TEXT + FRAME, before=(0, 300)),
        # a token of each of 32 samples over a prompt with eleven frames
        _case("token_32_samples", "attend", 32, page=32, prefix=TEXT + 11 * FRAME, before=(0, FRAME)),
        # five tokens of each of 16 samples at once, 32 / 8 heads
        _case("few_16_samples", "attend", 16, heads=(32, 8, 128), page=16, prefix=9201, before=(1, 700), rows=(5, 5)),
        # a token of each of 128 samples over 24 frames, every sample with up to two frames of its own
        _case("token_128_samples", "attend", 128, prefix=TEXT + 24 * FRAME, before=(0, 2 * FRAME)),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    small = rng.random() < 0.15
    heads = rng.choice([(4, 2, 64), (9, 3, 64)]) if small else rng.choice([(24, 8, 128), (24, 8, 128), (32, 8, 128), (16, 4, 128), (8, 8, 128), (24, 12, 128)])
    dtype = rng.choice(["f32", "bf16"]) if small else "bf16"
    page = rng.choice([16, 32, 64, 128])
    op = rng.choice(["append", "prompt", "prompt", "shared", "shared", "shared"])
    more = dict(heads=heads, dtype=dtype, page=page)
    if op == "append":
        seqs = _log_int(rng, 1, 64)
        hi = _log_int(rng, 1, 20000 // seqs)
        return _case("", op, seqs, before=(0, _log_int(rng, 1, 3000)), rows=(rng.randint(1, hi), hi), **more)
    if op == "prompt":
        seqs = _log_int(rng, 1, 24)
        hi = _log_int(rng, 16, max(20, min(8000, 12000 // seqs) // (4 if small else 1)))
        lo = rng.randint(1, hi)
        if rng.random() < 0.3:                 # a frame, or a prompt's next piece, over what is there
            return _case("", "attend", seqs, prefix=_log_int(rng, 1, 2000), before=(0, _log_int(rng, 1, 2000)), rows=(lo, min(hi, 1008)) if lo <= 1008 else (1008, 1008),
                         causal=rng.random() < 0.5, **more)
        return _case("", "attend", seqs, rows=(lo, hi), **more)
    seqs = _log_int(rng, 2, 128)
    rows = rng.choice([1, 1, 1, 2, 5, 8])
    if seqs * rows > 160:
        rows = 1
    most = 24000 if seqs <= 64 else 12000
    return _case("", "attend", seqs, prefix=_log_int(rng, 16, most // (4 if small else 1)), before=(0, _log_int(rng, 1, 2000)), rows=(rows, rows), **more)


def _lengths(c):
    """(rows, own tokens with the rows) of every sequence, by the case alone; the ranges' ends are among them where there is more than one sequence"""
    rng = random.Random("%d %d %d %d %d %d" % tuple(c[k] for k in ("seqs", "before_lo", "before_hi", "rows_lo", "rows_hi", "prefix")))
    rows = [rng.randint(c["rows_lo"], c["rows_hi"]) for _ in range(c["seqs"])]
    before = [rng.randint(c["before_lo"], c["before_hi"]) for _ in range(c["seqs"])]
    rows[0], before[-1] = c["rows_hi"], c["before_hi"]
    if c["seqs"] > 1:
        rows[-1], before[0] = c["rows_lo"], c["before_lo"]
    return rows, [b + r for b, r in zip(before, rows)]


# ---------------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------------
def _axes(d):
    """axis (0, 1, 2) and frequency of each rotary pair"""
    i = np.arange(d // 2)
    axis = i % 3
    n_axis = np.array([(axis == a).sum() for a in range(3)])
    return axis, BASE ** (-(i // 3) / n_axis[axis])


def _table(d):
    """[positions][pairs] (cos, sin) of position x frequency, and the pairs' axes"""
    axis, freq = _axes(d)
    ang = np.arange(max(MAX_POS), dtype=np.float64)[:, None] * freq
    return torch.from_numpy(np.stack([np.cos(ang), np.sin(ang)], -1).astype(np.float32)).cuda(), torch.from_numpy(axis).cuda()


def _rotate(tab, x, pos):
    """Rows [..., heads, d] in fp32 at positions [..., 4]"""
    t, axis = tab
    cs = t[pos[..., :3].long()[..., axis], torch.arange(len(axis), device=x.device)][..., None, :, :]
    x0, x1, c, s = x[..., 0::2], x[..., 1::2], cs[..., 0], cs[..., 1]
    return torch.stack([x0 * c - x1 * s, x0 * s + x1 * c], -1).flatten(-2)


def _positions(j):
    """(t, h, w, tag) of token j of a sequence: text, then frames"""
    f, r = (j - TEXT).div(FRAME, rounding_mode="floor"), (j - TEXT) % FRAME
    text = j < TEXT
    return torch.stack([torch.where(text, j, TEXT + 4 * f), torch.where(text, j, 8 * (r // COLS)), torch.where(text, j, 8 * (r % COLS)), j], -1).int()


class _State:
    pass


def _inputs(c, seed):
    """The tensors of a case from the seed alone."""
    s = _State()
    gen = torch.Generator(device="cuda").manual_seed(int(seed) % (1 << 62))
    dev = dict(device="cuda")
    hq, hkv, d, page, n = c["q_heads"], c["kv_heads"], c["head_dim"], c["page"], c["seqs"]
    dt = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
    rows, length = _lengths(c)
    starts = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
    total = int(starts[-1])
    s.n_rows, s.max_rows, s.max_own = total, max(rows), max(length)
    s.row_start, s.length = torch.from_numpy(starts).cuda(), torch.tensor(length, dtype=torch.int32, **dev)
    # which sequence a row is of, and the token that it is
    s.seq = torch.repeat_interleave(torch.arange(n, **dev), torch.tensor(rows, **dev))
    s.slot = torch.arange(total, **dev) - s.row_start[:-1].long()[s.seq] + (s.length.long() - torch.tensor(rows, **dev))[s.seq]
    s.pos = _positions(s.slot + c["prefix"]).contiguous()
    bias = torch.zeros(2, hkv * d, **dev)
    if c["dtype"] == "bf16":
        for b in bias:
            at = torch.randperm(hkv * d, generator=gen, **dev)[: max(1, hkv * d // 50)]
            b[at] = 4.0 * (1 - 2 * torch.randint(0, 2, at.shape, generator=gen, **dev).float())
    bias = bias.view(2, hkv, d)
    own_pages = [-(-m // page) for m in length]
    prefix_pages = -(-c["prefix"] // page)
    s.n_pages = sum(own_pages) + prefix_pages + 2
    order = torch.randperm(s.n_pages, generator=gen, **dev).int()
    s.prefix = order[:prefix_pages].contiguous()
    s.table = torch.zeros(n, max(own_pages), dtype=torch.int32, **dev)
    flat = order[prefix_pages:]
    ends = np.cumsum(own_pages)
    index = torch.arange(max(own_pages), **dev)[None]
    count, first = torch.tensor(own_pages, **dev)[:, None], torch.tensor(ends - own_pages, **dev)[:, None]
    s.table = torch.where(index < count, flat[(first + index).clamp(max=len(flat) - 1)], 0).int().contiguous()
    s.tab = _table(d)

    def pool(which):
        return (torch.randn(s.n_pages, page, hkv, d, generator=gen, **dev) + bias[which]).to(dt)

    s.k_pool, s.v_pool = pool(0), pool(1)
    if c["op"] == "append":
        s.k, s.v = ((torch.randn(total, hkv, d, generator=gen, **dev) + b).to(dt) for b in bias)
    else:
        s.q = torch.randn(total, hq, d, generator=gen, **dev).to(dt)
    return s


def prepare(case, seed):
    """Inputs, and what a program keeps beside them: the pool with what earlier steps put there, output buffers, workspaces."""
    c = dict(case)
    s = _inputs(c, seed)
    s.c, s.own = c, own
    if own:
        from paper_2601_04359_b200 import binding as pc
        s.ctx = pc.Context(c["q_heads"], c["kv_heads"], c["head_dim"], pc.PC_BF16 if c["dtype"] == "bf16" else pc.PC_F32, BASE, MAX_POS, s.n_rows, 1)
        s.pages = pc.Pages(s.k_pool, s.v_pool)
        s.batch = pc.Batch(s.table, s.length, s.row_start, s.max_rows, prefix=s.prefix if c["prefix"] else None, n_prefix=c["prefix"])
        if c["op"] == "attend":
            s.work = pc.PagedWork(s.ctx)
            s.out = torch.empty_like(s.q)
    return s


# ---------------------------------------------------------------------------------------------------------------------
# the plain form
# ---------------------------------------------------------------------------------------------------------------------
def _append(s):
    page = s.c["page"]
    at = s.table[s.seq, s.slot // page].long()
    s.k_pool[at, s.slot % page] = _rotate(s.tab, s.k.float(), s.pos).to(s.k.dtype)
    s.v_pool[at, s.slot % page] = s.v
    return {"k": s.k_pool, "v": s.v_pool}


def _attend(s):
    c = s.c
    n, hq, hkv, d = c["seqs"], c["q_heads"], c["kv_heads"], c["head_dim"]
    g, most = hq // hkv, s.max_rows
    start, rows = s.row_start[:-1].long(), (s.row_start[1:] - s.row_start[:-1]).long()
    i = torch.arange(most, device="cuda")
    at = (start[:, None] + i).clamp(max=s.n_rows - 1)                                                  # [n][most] rows, the last ones not there
    q = _rotate(s.tab, s.q.float(), s.pos)[at] * (1.0 / math.sqrt(d))                                  # [n][most][hq][d]
    q = q.view(n, most, hkv, g, d).permute(0, 2, 1, 3, 4).reshape(n, hkv, most * g, d)
    length = s.length.long()
    seen = (length - rows)[:, None] + i + 1 if c["causal"] else length[:, None].expand(n, most)        # own tokens that a row sees
    slots = s.table.shape[1] * c["page"]
    ko, vo = (x[s.table.long()].view(n, slots, hkv, d)[:, : s.max_own].float().permute(0, 2, 1, 3) for x in (s.k_pool, s.v_pool))
    x = torch.matmul(q, ko.transpose(-1, -2))
    hidden = torch.arange(s.max_own, device="cuda") >= seen.repeat_interleave(g, 1)[..., None]         # [n][most g][own]
    x.masked_fill_(hidden[:, None], -math.inf)
    m = x.amax(-1, keepdim=True)
    if c["prefix"]:
        kp, vp = (x[s.prefix.long()].view(-1, hkv, d)[: c["prefix"]].float().permute(1, 0, 2) for x in (s.k_pool, s.v_pool))
        shared = q.permute(1, 0, 2, 3).reshape(hkv, -1, d)                                             # the rows of all sequences at once
        y = torch.matmul(shared, kp.transpose(-1, -2))
        my = y.amax(-1).view(hkv, n, -1).permute(1, 0, 2)[..., None]
        m = torch.maximum(m, my)
        e = torch.exp(y - m.permute(1, 0, 2, 3).reshape(hkv, -1, 1))
        back = lambda z: z.view(hkv, n, most * g, -1).permute(1, 0, 2, 3)                              # noqa: E731
        total, out = back(e.sum(-1, keepdim=True)), back(torch.matmul(e, vp))
        e = x.sub_(m).exp_()
        total = total + e.sum(-1, keepdim=True)
        out = out + torch.matmul(e, vo)
    else:
        e = x.sub_(m).exp_()
        total, out = e.sum(-1, keepdim=True), torch.matmul(e, vo)
    out = (out / total).view(n, hkv, most, g, d).permute(0, 2, 1, 3, 4).reshape(n, most, hq, d)
    return {"out": out[s.seq, torch.arange(s.n_rows, device="cuda") - start[s.seq]].to(s.q.dtype)}


# ---------------------------------------------------------------------------------------------------------------------
# the calls that a user makes
# ---------------------------------------------------------------------------------------------------------------------
def _library(s):
    from paper_2601_04359_b200 import binding as pc
    if s.c["op"] == "append":
        pc.pc_paged_append(s.ctx, s.pages, s.batch, s.k, s.v, s.pos)
        return {"k": s.k_pool, "v": s.v_pool}
    pc.pc_paged_attend(s.work, s.pages, s.batch, s.q, s.pos, causal=s.c["causal"], out=s.out)
    return {"out": s.out}


def run(state):
    if state.own:
        return _library(state)
    return _append(state) if state.c["op"] == "append" else _attend(state)


# ---------------------------------------------------------------------------------------------------------------------
# work, and the definition in 64 bits
# ---------------------------------------------------------------------------------------------------------------------
def work(case):
    c = case
    hq, hkv, d = c["q_heads"], c["kv_heads"], c["head_dim"]
    elem = 2 if c["dtype"] == "bf16" else 4
    rows, length = _lengths(c)
    total, token = sum(rows), 2 * hkv * d * elem                       # bytes of a token's keys and values
    tables = 4 * (sum(-(-m // c["page"]) for m in length) + 2 * c["seqs"] + 1 + -(-c["prefix"] // c["page"]))
    if c["op"] == "append":
        return {"bytes": total * (2 * token + 16) + tables, "flops": total * hkv * d * 3}
    pairs = sum(r * c["prefix"] + (r * m - r * (r - 1) // 2 if c["causal"] else r * m) for r, m in zip(rows, length))
    return {"bytes": (sum(length) + c["prefix"]) * token + total * (2 * hq * d * elem + 16) + tables, "flops": 4 * hq * d * pairs}


def _turn(d, x, pos):
    """The rotary embedding as a product of complex numbers"""
    axis, freq = _axes(d)
    ang = pos[:, :3].double()[:, torch.from_numpy(axis).cuda()] * torch.from_numpy(freq).cuda()
    z = torch.view_as_complex(x.double().reshape(*x.shape[:-1], -1, 2).contiguous())
    return torch.view_as_real(z * torch.polar(torch.ones_like(ang), ang)[:, None, :]).flatten(-2)


def exact(case, seed):
    c = dict(case)
    s = _inputs(c, seed)
    hq, hkv, d, page = c["q_heads"], c["kv_heads"], c["head_dim"], c["page"]
    rows, length = _lengths(c)
    starts = np.concatenate([[0], np.cumsum(rows)])
    if c["op"] == "append":
        k, v = s.k_pool.double(), s.v_pool.double()
        turned = _turn(d, s.k, s.pos)
        for i, (r, m) in enumerate(zip(rows, length)):
            tokens = torch.arange(m - r, m, device="cuda")
            at = s.table[i].long()[tokens // page] * page + tokens % page
            k.view(-1, hkv, d)[at] = turned[starts[i]: starts[i + 1]]
            v.view(-1, hkv, d)[at] = s.v[starts[i]: starts[i + 1]].double()
        return {"k": k, "v": v}
    q = _turn(d, s.q, s.pos)
    out = torch.empty(s.n_rows, hq, d, dtype=torch.float64, device="cuda")
    kf, vf = s.k_pool.view(-1, hkv, d), s.v_pool.view(-1, hkv, d)
    in_page = torch.arange(page, device="cuda")
    prefix = (s.prefix.long()[:, None] * page + in_page).flatten()[: c["prefix"]]
    for i, (r, m) in enumerate(zip(rows, length)):
        tokens = torch.cat([prefix, (s.table[i].long()[:, None] * page + in_page).flatten()[:m]])
        k, v = kf[tokens].double(), vf[tokens].double()
        last = torch.arange(c["prefix"] + m - r, c["prefix"] + m, device="cuda")[:, None]
        hidden = torch.arange(len(tokens), device="cuda")[None] > (last if c["causal"] else torch.full_like(last, len(tokens)))
        for h in range(hq):
            x = q[starts[i]: starts[i + 1], h] @ k[:, h * hkv // hq].T / math.sqrt(d)
            p = torch.softmax(x.masked_fill_(hidden, -math.inf), 1)
            out[starts[i]: starts[i + 1], h] = p @ v[:, h * hkv // hq]
    return {"out": out}
