"""The paged cache where it can go wrong: infinities and NaN among hidden values, tables and lengths that make no sense, replayed graphs, other streams, waits that run out, pools
beyond 32-bit offsets, and a generation loop of several samples."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from paper_2601_04359_b200 import binding as pc
from tests.paged_reference import Paged, compare, turn

pytestmark = pytest.mark.gpu


def _bits(t):
    return t.view(torch.int16 if t.element_size() == 2 else torch.int32)


# the few-row kernel, the tcgen05 kernel, and both with a prefix
ROUTES = {"shared": ([5, 3, 1] + [1] * 60, [21, 3, 40] + [9] * 60, 1000), "few": ([5, 3, 1], [21, 3, 40], 0), "few_shared": ([5, 3, 1], [21, 3, 40], 37), "many": ([140, 60], [200, 60], 0), "many_prefix": ([140, 60], [200, 60], 50)}


@pytest.mark.parametrize("route", list(ROUTES))
@pytest.mark.parametrize("shape", ["lumos", "mha", "one", "small", "tiny_f32"])
@pytest.mark.parametrize("what", [float("inf"), float("-inf"), float("nan")])
def test_infinite_values_reach_the_rows_that_see_them(shape, route, what):
    rows, length, prefix = ROUTES[route]
    c = Paged(shape, rows, length, prefix=prefix)
    # among the last tokens of the first sequence, which its earlier rows do not see; and one that all of them see
    at = c.slots(0)
    v = c.v.view(-1, c.hkv, c.d)
    for back, head, channel in ((1, 0, 3), (2, c.hkv - 1, 5), (3, 0, c.d - 1), (length[0], 0, 8)):
        v[at[length[0] - back], head, channel] = what
    c.up()
    work = pc.PagedWork(c.ctx)
    want = c.want()
    assert (~want[0][: rows[0]].isfinite()).any()
    compare(c.attend(work), want)
    # a key that is NaN makes NaN of the rows that see it, and of no other
    c.k.view(-1, c.hkv, c.d)[at[length[0] - 2], 0] = float("nan")
    c.up()
    compare(c.attend(work), c.want())
    assert pc.pc_poll_status(c.ctx) == pc.PC_OK


@pytest.mark.parametrize("impl", [0, 1])
@pytest.mark.parametrize("shape", ["lumos", "small"])
def test_either_kernel_takes_prompts(shape, impl):
    c = Paged(shape, [200, 1, 77], [200, 90, 300], prefix=33, page=32)
    pc.pc_set_attend_impl(c.ctx, impl)
    compare(c.attend(pc.PagedWork(c.ctx)), c.want())


@pytest.mark.parametrize("rows,prefix", [(1, 100), (3, 40)])
def test_most_sequences(rows, prefix):
    """1,536 rows of 512 sequences are too many for a prefix of its own: every sequence reads it."""
    n = pc.PC_MAX_SEQS
    c = Paged("small", [rows] * n, [rows + i % 50 for i in range(n)], prefix=prefix)
    compare(c.attend(pc.PagedWork(c.ctx)), c.want())
    assert pc.pc_poll_status(c.ctx) == pc.PC_OK


def test_nothing_at_all():
    c = Paged("lumos", [0, 0], [7, 0])
    work = pc.PagedWork(c.ctx)
    out, lse = c.attend(work)
    assert out.shape[0] == 0
    pc.pc_paged_append(c.ctx, c.pages, c.batch, c.gpu["k_new"], c.gpu["v_new"], c.gpu["pos"])
    none = pc.Batch(c.table[:0].cuda(), torch.empty(0, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda"), 4)
    q = torch.full((3, 24, 128), 2.0, device="cuda").bfloat16()
    d = Paged("lumos", [3], [3])
    out = torch.full_like(q, 5.0)
    pc.pc_paged_attend(pc.PagedWork(d.ctx), d.pages, none, q, d.gpu["pos"], out=out)
    assert (out == 5).all() and pc.pc_poll_status(c.ctx) == pc.PC_OK


def _flawed(kind, c):
    """Makes sequence 1 of three senseless"""
    last = (c.length[1] - 1) // c.page                    # the entry that an append needs as well
    if kind == "page":
        c.table[1, last] = len(c.k)
    elif kind == "negative_page":
        c.table[1, last] = -1
    elif kind == "length":
        c.length[1] = c.table.shape[1] * c.page + 1
    elif kind == "negative_length":
        c.length[1] = -3
    elif kind == "rows":
        c.starts = c.starts.copy()
        c.starts[2] = c.starts[1] - 1
    elif kind == "position":
        c.pos[c.starts[1], 1] = 10 ** 6
    c.up()


@pytest.mark.parametrize("kind", ["page", "negative_page", "length", "negative_length", "rows", "position"])
@pytest.mark.parametrize("rows", [(2, 1, 2), (90, 40, 60)])
@pytest.mark.parametrize("prefix", [0, 20])
def test_senseless_numbers_are_recorded(kind, rows, prefix):
    length = [r + 20 for r in rows]
    good = Paged("lumos", rows, length, prefix=prefix)
    want = good.want()
    work = pc.PagedWork(good.ctx)
    compare(good.attend(work), want)
    c = Paged("lumos", rows, length, prefix=prefix, ctx=good.ctx)
    _flawed(kind, c)
    out, lse = c.attend(work)
    assert pc.pc_poll_status(c.ctx) == pc.PC_ERR_INVALID_ARG
    last = slice(int(good.starts[2]), None) if kind != "rows" else slice(int(good.starts[2]), int(good.starts[2]))       # (with the rows' starts, what follows is another sequence's as well)
    first = slice(0, rows[0] - (1 if kind == "rows" else 0))
    for part in (first, last):
        compare((out[part], lse[part]), [x[part] for x in want])
    # an append leaves the flawed one out, or turns its row at the nearest position, and nothing else changes
    k0 = c.pages.k.clone()
    pc.pc_paged_append(c.ctx, c.pages, c.batch, c.gpu["k_new"], c.gpu["v_new"], c.gpu["pos"])
    assert pc.pc_poll_status(c.ctx) == pc.PC_ERR_INVALID_ARG
    if kind in ("length", "negative_length", "rows"):
        at = good.slots(1).cuda()
        assert torch.equal(_bits(c.pages.k.view(-1, 8, 128)[at]), _bits(k0.view(-1, 8, 128)[at]))
    compare(good.attend(work), want)
    assert pc.pc_poll_status(c.ctx) == pc.PC_OK


@pytest.mark.parametrize("rows,prefix,length", [((1, 1, 1, 1), 70, (5, 30, 1, 64)), ((40, 100, 3, 1), 33, (40, 120, 60, 1)), ((1,) * 50, 1000, tuple(1 + i % 60 for i in range(50)))])
def test_a_captured_step_replays_with_other_numbers(rows, prefix, length):
    c = Paged("lumos", rows, length, prefix=prefix, page=16, free=0.0)
    work = pc.PagedWork(c.ctx)
    out = torch.empty_like(c.gpu["q"])

    def step():
        pc.pc_paged_append(c.ctx, c.pages, c.batch, c.gpu["k_new"], c.gpu["v_new"], c.gpu["pos"])
        pc.pc_paged_attend(work, c.pages, c.batch, c.gpu["q"], c.gpu["pos"], out=out)

    k0, v0 = c.pages.k.clone(), c.pages.v.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for turn_ in range(2):
        # other lengths, pages, rows and queries, in place
        d = Paged("lumos", rows[::-1] if turn_ else rows, length[::-1] if turn_ else [max(r, m - 1) for r, m in zip(rows, length)], prefix=prefix, page=16, seed=9 + turn_, ctx=c.ctx, free=0.0)
        c.batch.length.copy_(d.batch.length)
        c.batch.row_start.copy_(d.batch.row_start)
        c.batch.prefix.copy_(d.batch.prefix)
        c.batch.table.fill_(0)
        c.batch.table[:, : d.table.shape[1]] = d.batch.table[:, : c.table.shape[1]]
        n = min(len(k0), len(d.k))
        for mine, other in ((c.pages.k, d.k), (c.pages.v, d.v)):
            mine[:n] = other[:n].cuda()
        assert len(d.k) <= len(k0)
        for name in ("q", "k_new", "v_new", "pos"):
            c.gpu[name].copy_(d.gpu[name])
        graph.replay()
        got = out.clone()
        pc.pc_paged_append(d.ctx, d.pages, d.batch, d.gpu["k_new"], d.gpu["v_new"], d.gpu["pos"])
        want = pc.pc_paged_attend(work, d.pages, d.batch, d.gpu["q"], d.gpu["pos"])
        assert torch.equal(_bits(got), _bits(want))
        # and in 64 bits, over what the append has left
        d.k, d.v = d.pages.k.cpu(), d.pages.v.cpu()
        full = pc.pc_paged_attend(work, d.pages, d.batch, d.gpu["q"], d.gpu["pos"], want_lse=True)
        compare(full, d.want())
    assert pc.pc_poll_status(c.ctx) == pc.PC_OK


def test_another_stream():
    c = Paged("lumos", [1] * 6, [40, 3, 9, 100, 1, 17], prefix=90)
    work = pc.PagedWork(c.ctx)
    want = c.want()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = c.attend(work, stream=side)
    side.synchronize()
    compare(got, want)


@pytest.mark.parametrize("rows,prefix", [((1, 1), 0), ((1,) * 40, 1000), ((90, 40), 0)])
def test_waits_that_run_out(rows, prefix):
    c = Paged("lumos", rows, [r + 30 for r in rows], prefix=prefix)
    work = pc.PagedWork(c.ctx)
    before, lse = c.attend(work)
    pc.pc_set_wait_limit_us(c.ctx, 2000)
    pc.pc_test_expect_extra_bytes(c.ctx, 16)
    c.attend(work)
    assert pc.pc_poll_status(c.ctx) == pc.PC_ERR_TIMEOUT
    pc.pc_test_expect_extra_bytes(c.ctx, 0)
    pc.pc_set_wait_limit_us(c.ctx, 0)
    after, _ = c.attend(work)
    assert pc.pc_poll_status(c.ctx) == pc.PC_OK
    assert torch.equal(_bits(before), _bits(after))
    compare((after, lse), c.want())


def test_pages_beyond_32_bit_offsets():
    """Pools of 4.5 GB, of which the last pages are used."""
    n_pages, page = 17300, 128
    c = Paged("lumos", [1, 70, 1], [300, 70, 5], prefix=64, page=page)
    used = len(c.k)
    shift = n_pages - used
    big = [torch.empty(n_pages, page, 8, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    assert big[0].numel() * 2 > 2 ** 32
    for pool, mine in zip(big, (c.k, c.v)):
        pool[shift:] = mine.cuda()
    want, work = c.want(), pc.PagedWork(c.ctx)
    c.table += shift
    c.prefix = c.prefix + shift
    c.up()
    c.pages = pc.Pages(*big)
    compare(c.attend(work), want)
    pc.pc_paged_append(c.ctx, c.pages, c.batch, c.gpu["k_new"], c.gpu["v_new"], c.gpu["pos"])
    at = c.slots(1).cuda()
    got = big[1].view(-1, 8, 128)[at]
    assert torch.equal(_bits(got.cpu()), _bits(c.v_new[1:71])) and pc.pc_poll_status(c.ctx) == pc.PC_OK


@pytest.mark.parametrize("shape", ["lumos", "tiny_f32"])
def test_samples_of_a_prompt(shape):
    """A prompt enters the cache and attends to itself; then four samples of it go on by a piece, a token each and a frame, every step against 64 bits over all that was appended."""
    n_prompt, page = 70, 16
    prompt = Paged(shape, [n_prompt], [n_prompt], page=page, free=0.0, max_q=200)
    work = pc.PagedWork(prompt.ctx)
    pool = pc.Pages(*(torch.full((80, page, prompt.hkv, prompt.d), float("nan"), dtype=prompt.dtype, device="cuda") for _ in range(2)))
    prefix = torch.randperm(80, generator=torch.Generator().manual_seed(1)).int()
    pages = prefix[5:]
    prefix = prefix[:5].contiguous()
    rng = np.random.default_rng(3)
    held = torch.zeros(4, dtype=torch.int32)
    table = pages[:72].view(4, 18).contiguous()

    def step(rows, causal, n_prefix, own_table):
        c = Paged(shape, rows, rows, page=page, seed=int(rng.integers(1 << 20)), ctx=prompt.ctx, free=0.0)
        n = len(rows)
        length = torch.tensor(rows, dtype=torch.int32) if n_prefix == 0 else held + torch.tensor(rows, dtype=torch.int32)
        c.batch = pc.Batch(own_table.cuda(), length.cuda(), torch.from_numpy(c.starts).int().cuda(), max(rows), prefix=prefix.cuda() if n_prefix else None, n_prefix=n_prefix)
        pc.pc_paged_append(c.ctx, pool, c.batch, c.gpu["k_new"], c.gpu["v_new"], c.gpu["pos"])
        c.pages = pool
        got = c.attend(work, causal)
        c.k, c.v, c.table, c.prefix, c.n_prefix, c.length = pool.k.cpu(), pool.v.cpu(), own_table, prefix, n_prefix, length.tolist()
        compare(got, c.want(causal))
        # what the append has written is the rotated keys
        i0, at = int(c.starts[n - 1]), c.slots(n - 1)[-rows[-1]:]
        x = turn(c.k_new[i0:i0 + rows[-1]], c.pos[i0:i0 + rows[-1]])
        assert ((c.k.view(-1, c.hkv, c.d)[at].double() - x).abs() <= x.abs().clamp(min=1.0) * (2.0 ** -7 if c.dtype == torch.bfloat16 else 2.0 ** -20)).all()
        if n_prefix:
            held.add_(torch.tensor(rows, dtype=torch.int32))

    step([n_prompt], True, 0, prefix[None].contiguous())
    step([9, 33, 1, 20], True, n_prompt, table)
    for _ in range(3):
        step([1, 1, 1, 1], True, n_prompt, table)
    step([40, 40, 40, 40], False, n_prompt, table)
    step([2, 0, 1, 5], True, n_prompt, table)
    assert pc.pc_poll_status(prompt.ctx) == pc.PC_OK


@pytest.mark.parametrize("shape,most", [("tiny_f32", 2**31 - 1), ("tiny_f32", 6), ("lumos", 2**31 - 1), ("lumos", 6)])
def test_a_loose_bound_of_rows(shape, most):
    c = Paged(shape, [5, 1, 3], [21, 40, 3], prefix=37)
    want = c.want()
    c.batch.max_rows = most
    work = pc.PagedWork(c.ctx)
    compare(c.attend(work), want)
    assert pc.pc_poll_status(c.ctx) == pc.PC_OK


@pytest.mark.parametrize("prefix,rows", [(20011, [8]), (3001, [1, 1, 1, 1]), (0, [500, 90])])
def test_fp32_sums_do_not_drift(prefix, rows):
    """The error's norm over the output's.  Scores are a few units and sums of 8 rounded terms of 16 channels: 2^-24 x 4 x 3 (root of 8) / 2 on the way; exponential 2^-22, its argument
    2^-24 x 4; long sums of at most 50 rounded terms, errors of either sign: 2^-24 x 7.  Their root of squares is below 2^-20.8; sums that are cut off, six times a step, pass it."""
    c = Paged("lumos_f32", rows, [r + 40 if prefix else r for r in rows], prefix=prefix, page=64)
    out, _ = c.attend(pc.PagedWork(c.ctx))
    want = c.want()[0]
    assert (out.double().cpu() - want).norm() <= 2.0 ** -20 * want.norm()


@pytest.mark.parametrize("shape,rows,prefix", [("lumos", [128], 2001), ("lumos", [100], 9000), ("gqa4", [50, 200, 1, 90], 2500), ("one", [60, 700], 1500), ("small", [40] * 9, 3000),
                                               ("lumos", [1400], 300)])
@pytest.mark.parametrize("causal", [True, False])
def test_few_pairs_over_many_tokens(shape, rows, prefix, causal):
    """Pairs of query tiles that leave SMs idle are cut along the keys, into parts that run at once"""
    c = Paged(shape, rows, [r + 70 for r in rows], prefix=prefix, page=32, behind=2)
    work = pc.PagedWork(c.ctx)
    got = c.attend(work, causal)
    compare(got, c.want(causal))
    again = c.attend(work, causal)
    assert torch.equal(_bits(again[0][:-2]), _bits(got[0][:-2])) and pc.pc_poll_status(c.ctx) == pc.PC_OK


def test_two_calls_at_once():
    """Two streams, a workspace each, one context: the same bits as one after the other"""
    a = Paged("lumos", [1] * 40, [1 + i % 30 for i in range(40)], prefix=1500, page=64, max_q=400)
    b = Paged("lumos", [140, 60], [200, 90], prefix=70, page=16, seed=5, ctx=a.ctx)
    calls = [(a, pc.PagedWork(a.ctx)), (b, pc.PagedWork(a.ctx))]
    alone = [c.attend(w)[0].clone() for c, w in calls]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in calls]
    got = [[], []]
    for _ in range(20):
        for i, (c, w) in enumerate(calls):
            with torch.cuda.stream(streams[i]):
                got[i].append(c.attend(w)[0])
    torch.cuda.synchronize()
    for i in range(2):
        for x in got[i]:
            assert torch.equal(_bits(x), _bits(alone[i]))
    assert pc.pc_poll_status(a.ctx) == pc.PC_OK
