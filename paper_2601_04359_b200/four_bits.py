"""A generation loop over a cache that is held in four bits and cut by accumulated attention weight (synthetic lumos-shaped layer).

    python -m paper_2601_04359_b200.four_bits [--frames 24] [--tokens 4] [--budget 8064] [--grid 24 42] [--heads 24 8] [--reps 10]

Per frame: the frame's queries attend anchors ++ history (pc_q4_attend), the finished frame's keys and values enter the history
(pc_q4_store), then a few text tokens are generated one at a time: each is stored and attends to everything so far, and the attention
it pays is added to the tokens' weights.  Once the history holds more than the budget, pc_q4_evict keeps the newest frame with its
text and the heaviest of the rest, packs them into the other of two buffers and shifts the time axis by one frame (Eq. 9).  One JSON line:
times of a frame step, a token and an eviction (CUDA events over repeated calls on the final cache), bytes of the cache in four
and in 16 bits, and how far the last token's output is from 16-bit attention over the same tokens read back."""
from __future__ import annotations

import argparse
import json

import torch

from . import binding as pc

T_STEP = 4


def _positions(n_text, t, rows, cols, tag):
    i = torch.arange(rows * cols, dtype=torch.int32, device="cuda")
    return torch.stack([torch.full_like(i, n_text + T_STEP * t), 8 * (i // cols), 8 * (i % cols), tag + i], 1).contiguous()


def _time(fn, reps):
    for _ in range(3):
        fn()
    a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    torch.cuda.synchronize()
    a.record()
    for _ in range(reps):
        fn()
    b.record()
    torch.cuda.synchronize()
    return a.elapsed_time(b) / reps * 1e3


def generate(frames=24, tokens=4, budget=8064, grid=(24, 42), heads=(24, 8), n_text=128, decay=0.98, reps=10, seed=0):
    """Runs the loop; returns what the command prints."""
    hq, hkv = heads
    d, n = 128, grid[0] * grid[1]
    gen = torch.Generator(device="cuda").manual_seed(seed)
    bias = torch.zeros(2, hkv * d, device="cuda")
    for b in bias:                                       # channel outliers, as trained layers have them
        b[torch.randperm(hkv * d, generator=gen, device="cuda")[: hkv * d // 50]] = 4.0
    bias = bias.view(2, hkv, d)

    def rows(count, pos):
        k, v = (torch.randn(count, hkv, d, generator=gen, device="cuda") + b for b in bias)
        return pc.Segment(k.bfloat16(), v.bfloat16(), pos, count)

    def queries(count):
        return torch.randn(count, hq, d, generator=gen, device="cuda").bfloat16()

    step = n + tokens                                    # tokens that a frame and its text add
    capacity = budget + 2 * step
    n_anchor = n_text + n
    ctx = pc.Context(hq, hkv, d, pc.PC_BF16, 10000.0, (n_text + T_STEP * (frames + 2), max(n_text, 8 * grid[0]), max(n_text, 8 * grid[1])),
                     n, n_anchor + capacity)
    work = pc.Q4Work(ctx, n_anchor + capacity, frames=True, weigh=True)
    text = torch.arange(n_text, dtype=torch.int32, device="cuda")[:, None].expand(n_text, 4).contiguous()
    anchors = pc.Q4Segment.empty(ctx, n_anchor)
    pc.pc_q4_store(ctx, rows(n_text, text), anchors)
    pc.pc_q4_store(ctx, rows(n, _positions(n_text, 0, *grid, n_text)), anchors)
    hist, other = (pc.Q4Segment.empty(ctx, capacity, weight=True) for _ in range(2))
    evictions = 0
    for f in range(1, frames + 1):
        t = f - hist.t_shift // T_STEP                   # in the shifted frame of reference
        cache = pc.Q4Cache(anchors, hist)
        pos = _positions(n_text, t, *grid, n_anchor + (f - 1) * step)
        pc.pc_q4_attend(work, cache, queries(n), pos)
        pc.pc_q4_store(ctx, rows(n, pos), hist)
        for i in range(tokens):
            at = torch.tensor([[n_text + T_STEP * t, 0, 0, n_anchor + (f - 1) * step + n + i]], dtype=torch.int32, device="cuda")
            q = queries(1)
            pc.pc_q4_store(ctx, rows(1, at), hist)
            out = pc.pc_q4_attend(work, cache, q, at, weigh=(decay, 1.0))
        if f < frames and hist.n_tokens > budget:
            pc.pc_q4_evict(ctx, hist, budget, min(step, budget), other, delta_t=T_STEP)
            hist, other = other, hist
            other.n_tokens, other.t_shift = 0, 0
            evictions += 1
    status = pc.pc_poll_status(ctx)
    assert status == pc.PC_OK, f"device status {status}"

    # the last token again, over the same tokens in 16 bits
    def thaw(seg):
        to = pc.Segment(*(torch.empty(seg.n_tokens, hkv, d, dtype=torch.bfloat16, device="cuda") for _ in range(2)),
                        torch.empty(seg.n_tokens, 4, dtype=torch.int32, device="cuda"), 0)
        pc.pc_q4_load(ctx, seg, 0, seg.n_tokens, to)
        return to

    a16, h16 = thaw(anchors), thaw(hist)
    want = pc.pc_attend_frame(ctx, pc.Cache(a16, h16, [h16.n_tokens]), None, q, at)
    off = float((out.float() - want.float()).abs().max())

    cache = pc.Q4Cache(anchors, hist)
    qn, one = queries(n), queries(1)
    scratch = pc.Q4Segment.empty(ctx, budget, weight=True)
    report = {"frames": frames, "history": hist.n_tokens, "evictions": evictions, "t_shift": hist.t_shift,
              "weight": float(hist.weight[:hist.n_tokens].sum()), "off_16bit": off,
              "bytes_4bit": (n_anchor + hist.n_tokens) * hkv * 5 * d // 4, "bytes_16bit": (n_anchor + hist.n_tokens) * hkv * 4 * d,
              "us_frame": _time(lambda: pc.pc_q4_attend(work, cache, qn, pos), reps),
              "us_token": _time(lambda: pc.pc_q4_attend(work, cache, one, at, weigh=(decay, 1.0)), reps),
              "us_evict": _time(lambda: pc.pc_q4_evict(ctx, hist, budget, min(step, budget), scratch, delta_t=T_STEP), reps)}
    work.close()
    ctx.close()
    return report


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--frames", type=int, default=24)
    ap.add_argument("--tokens", type=int, default=4)
    ap.add_argument("--budget", type=int, default=8064)
    ap.add_argument("--grid", type=int, nargs=2, default=(24, 42))
    ap.add_argument("--heads", type=int, nargs=2, default=(24, 8))
    ap.add_argument("--reps", type=int, default=10)
    args = ap.parse_args()
    if not torch.cuda.is_available():
        raise RuntimeError("the loop needs a CUDA device; there is no CPU fallback")
    print(json.dumps(generate(args.frames, args.tokens, args.budget, tuple(args.grid), tuple(args.heads), reps=args.reps)))


if __name__ == "__main__":
    main()
