"""The paged cache: rows appended with their rotation, and attention over it, against 64-bit restatements (tests/paged_reference.py has the tolerances)."""
from __future__ import annotations

import pytest
import torch

from paper_2601_04359_b200 import binding as pc
from tests.paged_reference import SHAPES, Paged, compare, turn

pytestmark = pytest.mark.gpu


def _bits(t):
    return t.view(torch.int16 if t.element_size() == 2 else torch.int32)


# rows, length with them
BATCHES = {"one_token": ([1], [1]), "ragged": ([3, 0, 17, 1, 40], [3, 9, 30, 100, 40]), "nothing_of_some": ([0, 0, 2, 0], [0, 5, 2, 0]),
           "odd_many": ([1 + i % 3 for i in range(37)], [5 + 7 * i for i in range(37)])}


@pytest.mark.parametrize("page", [16, 64, 128])
@pytest.mark.parametrize("batch", list(BATCHES))
@pytest.mark.parametrize("shape", ["lumos", "wide", "one", "odd64", "tiny_f32", "odd_f32", "lumos_f32"])
def test_append(shape, batch, page):
    rows, length = BATCHES[batch]
    c = Paged(shape, rows, length, page=page, behind=2)
    k0, v0 = c.k.clone(), c.v.clone()
    pc.pc_paged_append(c.ctx, c.pages, c.batch, c.gpu["k_new"], c.gpu["v_new"], c.gpu["pos"])
    assert pc.pc_poll_status(c.ctx) == pc.PC_OK
    k, v = (x.cpu().view(-1, c.hkv, c.d) for x in (c.pages.k, c.pages.v))
    written = torch.zeros(len(k), dtype=torch.bool)
    for s, (r, m) in enumerate(zip(rows, length)):
        at, i0 = c.slots(s)[m - r:], int(c.starts[s])
        written[at] = True
        x = c.k_new[i0:i0 + r]
        want = turn(x, c.pos[i0:i0 + r])
        pair = x.double().unflatten(-1, (x.shape[-1] // 2, 2)).abs().sum(-1).repeat_interleave(2, -1)
        # two products and a sum in fp32 with table entries of 24 bits, then half a unit of the type
        tol = pair * 2.0 ** -22 + want.abs() * (2.0 ** -8 if c.dtype == torch.bfloat16 else 2.0 ** -24)
        assert ((k[at].double() - want).abs() <= tol).all()
        assert torch.equal(_bits(v[at]), _bits(c.v_new[i0:i0 + r]))
    for x, before in ((k, k0), (v, v0)):                      # nothing else has changed
        assert torch.equal(_bits(x[~written]), _bits(before.view(-1, c.hkv, c.d)[~written]))


CASES = {
    # name: (rows, length, prefix, causal)
    "one_token": ([1], [1], 0, True),
    "tokens": ([1] * 5, [1, 15, 16, 17, 300], 0, True),
    "tokens_shared": ([1] * 5, [1, 15, 16, 17, 300], 37, True),
    "tokens_shared_long": ([1] * 33, [1 + 13 * i for i in range(33)], 1025, True),
    "few_shared": ([5, 0, 3, 1], [5, 4, 77, 130], 129, True),
    "many_tokens_shared": ([1 + (i == 7) for i in range(150)], [1 + i % 40 for i in range(150)], 700, True),
    "few_seeing_all": ([2, 1], [40, 3], 50, False),
    "prompts": ([1, 50, 129, 2, 257], [1, 50, 129, 2, 257], 0, True),
    "pieces": ([33, 100], [200, 101], 0, True),
    "pieces_shared": ([33, 100, 1], [200, 101, 1], 45, True),
    "frames": ([135, 135], [135, 405], 96, False),
    "frames_without_own": ([40, 40], [0, 300], 0, False),
    "more_rows_than_tokens": ([9, 30], [4, 30], 0, True),
    "only_a_prefix": ([1, 4], [0, 0], 66, False),
}


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("case", list(CASES))
@pytest.mark.parametrize("shape", list(SHAPES))
def test_attend(shape, case, page):
    rows, length, prefix, causal = CASES[case]
    c = Paged(shape, rows, length, prefix=prefix, page=page, behind=3)
    work = pc.PagedWork(c.ctx)
    out = torch.full_like(c.gpu["q"], 7.0)
    got = c.attend(work, causal, out=out)
    assert pc.pc_poll_status(c.ctx) == pc.PC_OK
    assert (out[-3:] == 7).all()
    compare(got, c.want(causal))
    again = c.attend(work, causal)
    assert torch.equal(_bits(again[0][:-3]), _bits(out[:-3]))


@pytest.mark.parametrize("shape,rows,length,prefix", [
    ("lumos", [1, 1], [3, 40], 25001),                 # six packed rows over a prefix that is read once
    ("lumos", [1, 1, 1, 1], [3, 1, 40, 17], 9001),     # twelve
    ("small", [1] * 150, [1 + i % 30 for i in range(150)], 2001),
    ("odd64", [2] * 100, [2 + i % 30 for i in range(100)], 1501),
    ("lumos", [5] * 40, [5 + i % 30 for i in range(40)], 1001),
    ("gqa4", [9] * 12, [9 + i for i in range(12)], 1001),
    ("tiny_f32", [1] * 80, [1 + i % 30 for i in range(80)], 1501),
    ("lumos_f32", [1] * 9, [1 + 7 * i for i in range(9)], 2001),
    ("lumos_f32", [3, 1, 4, 1, 5], [40, 3, 4, 50, 21], 2501),
])
def test_a_prefix_read_once(shape, rows, length, prefix):
    c = Paged(shape, rows, length, prefix=prefix, page=128, behind=3)
    work = pc.PagedWork(c.ctx)
    got = c.attend(work)
    compare(got, c.want())
    again = c.attend(work)
    assert torch.equal(_bits(again[0][:-3]), _bits(got[0][:-3])) and pc.pc_poll_status(c.ctx) == pc.PC_OK
