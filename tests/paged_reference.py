"""A paged batch for tests, and what the calls give in 64 bits, from the definition.

Tolerances.  A logit of a bf16 context is off by the one rounding of the rotated query, half a step of eight bits: delta = 2^-8 S with S = sum |R q| |k| / sqrt(d), and by what its fp32 sums
round: d / 16 instructions of 16 products, each off by no more than 2^-22 of S.  fp32 contexts have six instructions for every one and leave out
terms of 2^-24: delta = (6 d / 16 + 4) 2^-22 S.  The rotation itself (products with table entries of 24 bits) adds 2^-22 S.  A probability is then off by 2 delta relative (itself and the
normaliser) and 2^-18 (exponential, rescaling, sums of the normaliser), in bf16 by 2^-8 more where it is rounded for its product.  An output adds the roundings of its own sums, one for
every 16 keys (six in fp32), 2^-22 of sum p |v| each, and half a unit of its type."""
from __future__ import annotations

import numpy as np
import torch

from paper_2601_04359_b200 import binding as pc

BASE = 10000.0
MAX_POS = (600, 400, 400)
SHAPES = {"lumos": (24, 8, 128, "bf16"), "gqa4": (32, 8, 128, "bf16"), "mha": (8, 8, 128, "bf16"), "wide": (24, 12, 128, "bf16"), "one": (7, 1, 128, "bf16"),
          "group20": (20, 1, 128, "bf16"), "small": (4, 2, 64, "bf16"), "odd64": (9, 3, 64, "bf16"), "tiny_f32": (4, 2, 64, "f32"), "lumos_f32": (24, 8, 128, "f32"),
          "odd_f32": (5, 5, 64, "f32")}


def axes(d):
    i = np.arange(d // 2)
    axis = i % 3
    n_axis = np.array([(axis == a).sum() for a in range(3)])
    return torch.from_numpy(axis), torch.from_numpy(BASE ** (-(i // 3) / n_axis[axis]))


def turn(x, pos):
    """Rows [n][heads][d] rotated at positions [n][4], in 64 bits on the CPU"""
    axis, freq = axes(x.shape[-1])
    ang = pos[:, :3].double()[:, axis] * freq
    z = torch.view_as_complex(x.double().unflatten(-1, (x.shape[-1] // 2, 2)).contiguous())
    return torch.view_as_real(z * torch.polar(torch.ones_like(ang), ang)[:, None, :]).flatten(-2)


class Paged:
    """Sequences with rows[s] rows and length[s] tokens over a pool whose free places hold `free` (NaN: what nobody may read)."""

    def __init__(self, shape, rows, length, *, prefix=0, page=16, seed=0, behind=0, max_q=0, free=float("nan"), scale=1.0, ctx=None):
        self.hq, self.hkv, self.d, kind = SHAPES[shape]
        self.dtype = torch.bfloat16 if kind == "bf16" else torch.float32
        self.rows, self.length, self.n_prefix, self.page = list(rows), list(length), prefix, page
        gen = torch.Generator().manual_seed(seed + 7)
        starts = np.concatenate([[0], np.cumsum(rows)])
        self.starts, total = starts, int(starts[-1])
        own = [-(-m // page) for m in length]
        pre = -(-prefix // page)
        n_pages = sum(own) + pre + 2
        order = torch.randperm(n_pages, generator=gen).int()
        self.prefix = order[:pre]
        wide = max(own + [1])
        table = torch.full((len(rows), wide), 2 ** 30, dtype=torch.int32)      # entries that are not read name no page
        at = pre
        for s, n in enumerate(own):
            table[s, :n] = order[at:at + n]
            at += n
        self.table = table
        shape4 = (n_pages, page, self.hkv, self.d)
        self.k = torch.full(shape4, free).to(self.dtype)
        self.v = torch.full(shape4, free).to(self.dtype)
        used = torch.cat([self.slots(None)] + [self.slots(s) for s in range(len(rows))]).long()
        for x in (self.k, self.v):
            x.view(-1, self.hkv, self.d)[used] = (torch.randn(len(used), self.hkv, self.d, generator=gen) * scale).to(self.dtype)
        n = total + behind
        self.q = (torch.randn(n, self.hq, self.d, generator=gen) * scale).to(self.dtype)
        self.k_new, self.v_new = (torch.randn(n, self.hkv, self.d, generator=gen).to(self.dtype) for _ in range(2))
        self.pos = torch.stack([torch.randint(0, m, (n,), generator=gen) for m in MAX_POS] + [torch.arange(n)], 1).int()
        if behind:                                                              # rows that are nobody's: nothing of them is looked at
            self.pos[total:] = 10 ** 6
            self.q[total:] = float("nan")
        self.ctx = ctx or pc.Context(self.hq, self.hkv, self.d, pc.PC_BF16 if kind == "bf16" else pc.PC_F32, BASE, MAX_POS, max_q or max(n, 1), 1)
        self.up()

    def up(self):
        """To the GPU, as it is now."""
        self.pages = pc.Pages(self.k.cuda(), self.v.cuda())
        self.batch = pc.Batch(self.table.cuda(), torch.tensor(self.length, dtype=torch.int32).cuda(), torch.from_numpy(self.starts).int().cuda(), max(self.rows + [0]),
                              self.prefix.cuda() if self.n_prefix else None, self.n_prefix)
        self.gpu = {n: getattr(self, n).cuda() for n in ("q", "k_new", "v_new", "pos")}

    def slots(self, s):
        """Places in the pool of a sequence's own tokens (None: of the prefix)"""
        pages, n = (self.prefix, self.n_prefix) if s is None else (self.table[s], self.length[s])
        j = torch.arange(n)
        return pages[j // self.page].long() * self.page + j % self.page if n else torch.empty(0, dtype=torch.long)

    def attend(self, work, causal=True, **kw):
        return pc.pc_paged_attend(work, self.pages, self.batch, self.gpu["q"], self.gpu["pos"], causal=causal, want_lse=True, **kw)

    def want(self, causal=True):
        """(out, lse, tolerance of out, tolerance of lse) in 64 bits; rows that are nobody's are NaN"""
        n, d, g = len(self.q), self.d, self.hq // self.hkv
        out = torch.full((n, self.hq, d), float("nan"), dtype=torch.float64)
        lse, tol, tol_lse = out[..., 0].clone(), out.clone(), out[..., 0].clone()
        bf = self.dtype == torch.bfloat16
        ulp = (2.0 ** -8 + (d / 16 + 1) * 2.0 ** -22) if bf else (6 * d / 16 + 5) * 2.0 ** -22
        k, v = (x.view(-1, self.hkv, d).double() for x in (self.k, self.v))
        for s, (r, m) in enumerate(zip(self.rows, self.length)):
            at = torch.cat([self.slots(None), self.slots(s)])
            i0 = int(self.starts[s])
            if r == 0:
                continue
            q = turn(self.q[i0:i0 + r], self.pos[i0:i0 + r])
            ks, vs = (x[at].repeat_interleave(g, 1).permute(1, 0, 2) for x in (k, v))
            j = torch.arange(len(at))[None]
            seen = j < (self.n_prefix + ((m - r + 1 + torch.arange(r)[:, None]).clamp(min=0) if causal else torch.full((r, 1), m)))
            x = torch.einsum("ihd,hjd->hij", q, ks).div(d ** 0.5).masked_fill(~seen[None], float("-inf"))
            big = torch.einsum("ihd,hjd->hij", q.abs(), ks.abs()).div(d ** 0.5).masked_fill(~seen[None], 0.0)
            z = torch.logsumexp(x, -1) if len(at) else torch.full((self.hq, r), float("-inf"), dtype=torch.float64)
            p = torch.exp(x - z[..., None]).masked_fill(~seen[None], 0.0)
            delta = ulp * (big.amax(-1) if len(at) else torch.zeros_like(z))
            seen_v = lambda w: torch.stack([(p[:, i, :, None] * torch.where(seen[i][None, :, None], w, 0.0)).sum(1) for i in range(r)])     # noqa: E731
            o = seen_v(vs)
            spread = seen_v(vs.abs()) * (torch.expm1(2 * delta).T[..., None] + 2.0 ** -18 + (2.0 ** -8 if bf else 0.0) + (len(at) / 16 + 8) * (1 if bf else 6) * 2.0 ** -22)
            out[i0:i0 + r], lse[i0:i0 + r] = o, z.T
            tol[i0:i0 + r] = spread * 1.01 + o.abs() * (2.0 ** -8 if bf else 2.0 ** -24)
            tol_lse[i0:i0 + r] = (delta.T + 2.0 ** -18 * (1 + z.T.abs().nan_to_num(posinf=0.0))).nan_to_num()
        return out, lse, tol, tol_lse


def compare(got, want):
    """(out, lse) of a call against Paged.want(): what is infinite, NaN or empty exactly, the rest within the tolerance; rows that are nobody's are not looked at"""
    (out, lse), (o, z, tol, tol_lse) = got, want
    out, lse = out.double().cpu(), lse.double().cpu()
    mine = ~tol_lse.isnan().all(-1)
    out, lse, o, z, tol, tol_lse = (x[mine] for x in (out, lse, o, z, tol, tol_lse))
    empty = z == float("-inf")
    assert (out[empty] == 0).all() and (lse[empty] == float("-inf")).all()
    for x, w, t in ((out, o, tol), (lse, z, tol_lse)):
        fine = w.isfinite()
        assert torch.equal(x.isnan(), w.isnan()) and torch.equal(x[~fine & ~w.isnan()], w[~fine & ~w.isnan()])
        assert ((x - w).abs() <= t)[fine].all(), float(((x - w).abs() / t)[fine].max())
