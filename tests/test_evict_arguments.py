"""Eviction: what its callers hand over. Nothing at all, from nothing and into nothing."""
from __future__ import annotations

import pytest
import torch

from paper_2601_04359_b200 import binding as pc
from tests.test_q4_cache import _ctx


@pytest.mark.gpu
@pytest.mark.parametrize("room", [0, 5])
def test_nothing_is_kept_of_nothing(room):
    ctx = _ctx("lumos", 1, 64)
    dst = pc.Q4Segment.empty(ctx, room, weight=True)
    dst.n_tokens = room
    sel = pc.pc_q4_evict(ctx, pc.Q4Segment.empty(ctx, 0, t_shift=3), 5, 2, dst, delta_t=4)
    assert dst.n_tokens == 0 and dst.t_shift == 7 and sel.dtype == torch.int32 and sel.is_cuda
    for weight in (None, torch.empty(0, device="cuda")):
        to = pc.Segment(torch.empty(room, 8, 128, dtype=torch.bfloat16, device="cuda"), torch.empty(room, 8, 128, dtype=torch.bfloat16, device="cuda"),
                        torch.empty(room, 4, dtype=torch.int32, device="cuda"), room) if room else pc.Segment.empty()
        sel = pc.pc_evict(ctx, pc.Segment.empty(), weight, 5, 2, to)
        assert to.n_tokens == 0 and sel.is_cuda
    assert pc.pc_poll_status(ctx) == pc.PC_OK


# ---------------------------------------------------------------------------------------------------------------------
# types and lengths: looked at before the library is called, so a context that is closed is enough to see it
# ---------------------------------------------------------------------------------------------------------------------
class _Closed:
    handle = None
    sizes = (4, 2, 64, torch.float32)


class _Work:
    handle, ctx = None, _Closed


def _rows(n, dtype=torch.float32):
    return pc.Segment(torch.zeros(n, 2, 64, dtype=dtype), torch.zeros(n, 2, 64, dtype=dtype), torch.zeros(n, 4, dtype=torch.int32), n)


def _held(n, width=160):
    return pc.Q4Segment(torch.zeros(n, width, dtype=torch.uint8), torch.zeros(n, 4, dtype=torch.int32), torch.zeros(n), n)


def _with(x, **kw):
    for k, v in kw.items():
        setattr(x, k, v)
    return x


def _attend(cache=None, **kw):
    a = {"q": torch.zeros(3, 4, 64), "q_pos": torch.zeros(3, 4, dtype=torch.int32), "valid": torch.ones(6, dtype=torch.bool), "out": torch.zeros(3, 4, 64),
         "lse": torch.zeros(3, 4), **kw}
    return lambda: pc.pc_q4_attend(_Work, cache or pc.Q4Cache(_held(2), _held(6)), stream=0, **a)


def _evict(src=None, dst=None, **kw):
    a = {"weight": torch.zeros(6), "dst_weight": torch.zeros(4), "valid": torch.ones(6, dtype=torch.uint8), "sel_idx": torch.zeros(4, dtype=torch.int32), **kw}
    return lambda: pc.pc_evict(_Closed, src or _rows(6), a.pop("weight"), 4, 1, dst or _rows(4), stream=0, **a)


def _evict4(src=None, dst=None, **kw):
    a = {"valid": torch.ones(6, dtype=torch.uint8), "sel_idx": torch.zeros(4, dtype=torch.int32), **kw}
    return lambda: pc.pc_q4_evict(_Closed, src or _held(6), 4, 1, dst or _held(4), stream=0, **a)


I32 = torch.int32
REFUSED = {
    "rows of another context": (lambda: pc.pc_q4_store(_Closed, _rows(3), _held(6, 320), 0, stream=0), "rows has 1920 elements, 960 are needed"),
    "rows of another type": (lambda: pc.pc_q4_store(_Closed, _rows(3), _with(_held(6), rows=torch.zeros(6, 160)), 0, stream=0), "rows has to be torch.uint8"),
    "positions for fewer tokens": (lambda: pc.pc_q4_store(_Closed, _rows(3), _with(_held(6), pos=torch.zeros(5, 4, dtype=I32)), 0, stream=0), "pos has 20 elements, 24"),
    "weights for fewer tokens": (lambda: pc.pc_q4_store(_Closed, _rows(3), _with(_held(6), weight=torch.zeros(5)), 0, stream=0), "weight has 5 elements, 6"),
    "weights in 64 bits": (lambda: pc.pc_q4_store(_Closed, _rows(3), _with(_held(6), weight=torch.zeros(6).double()), 0, stream=0), "weight has to be torch.float32"),
    "keys in 16 bits": (lambda: pc.pc_q4_store(_Closed, _rows(3, torch.bfloat16), _held(6), 0, stream=0), "k has to be torch.float32"),
    "fewer values than keys": (lambda: pc.pc_q4_load(_Closed, _held(6), 0, 3, _with(_rows(3), v=torch.zeros(2, 2, 64)), stream=0), "v has 256 elements, 384"),
    "a short row of keys": (lambda: pc.pc_q4_load(_Closed, _held(6), 0, 3, _with(_rows(3), k=torch.zeros(3, 1, 64)), stream=0), "k has 192 elements, 384"),
    "a short mask": (_attend(valid=torch.ones(5, dtype=torch.bool)), "valid has 5 elements, 6"),
    "a mask of words": (_attend(valid=torch.ones(6, dtype=I32)), "valid has to be of one byte"),
    "queries of other heads": (_attend(q=torch.zeros(3, 2, 64)), "q has 384 elements, 768"),
    "queries in 16 bits": (_attend(q=torch.zeros(3, 4, 64, dtype=torch.bfloat16)), "q has to be torch.float32"),
    "fewer positions than queries": (_attend(q_pos=torch.zeros(2, 4, dtype=I32)), "q_pos has 8 elements, 12"),
    "positions in 64 bits": (_attend(q_pos=torch.zeros(3, 4, dtype=torch.int64)), "q_pos has to be torch.int32"),
    "a short output": (_attend(out=torch.zeros(2, 4, 64)), "out has 512 elements, 768"),
    "an output of another type": (_attend(out=torch.zeros(3, 4, 64, dtype=torch.bfloat16)), "out has to be torch.float32"),
    "a short lse": (_attend(lse=torch.zeros(3, 3)), "lse has 9 elements, 12"),
    "anchors of another context": (_attend(cache=pc.Q4Cache(_held(2, 80), _held(6))), "rows has 160 elements, 320"),
    "too few weights": (_evict(weight=torch.zeros(5)), "weight has 5 elements, 6"),
    "whole numbers as weights": (_evict(weight=torch.zeros(6, dtype=I32)), "weight has to be torch.float32"),
    "a short mask of an eviction": (_evict(valid=torch.ones(5, dtype=torch.uint8)), "valid has 5 elements, 6"),
    "too few indices": (_evict(sel_idx=torch.zeros(3, dtype=I32)), "sel_idx has 3 elements, 4"),
    "indices in 64 bits": (_evict(sel_idx=torch.zeros(4, dtype=torch.int64)), "sel_idx has to be torch.int32"),
    "too few new weights": (_evict(dst_weight=torch.zeros(3)), "dst_weight has 3 elements, 4"),
    "fewer positions than kept": (_evict(dst=_with(_rows(4), pos=torch.zeros(3, 4, dtype=I32))), "pos has 12 elements, 16"),
    "a short mask, four bits": (_evict4(valid=torch.ones(5, dtype=torch.uint8)), "valid has 5 elements, 6"),
    "too few indices, four bits": (_evict4(sel_idx=torch.zeros(3, dtype=I32)), "sel_idx has 3 elements, 4"),
    "too few weights, four bits": (_evict4(src=_with(_held(6), weight=torch.zeros(5))), "weight has 5 elements, 6"),
}


@pytest.mark.parametrize("case", list(REFUSED))
def test_what_does_not_fit_is_refused_by_name(case):
    call, text = REFUSED[case]
    with pytest.raises(pc.PackCacheError, match=text) as e:
        call()
    assert e.value.status == pc.PC_ERR_INVALID_ARG


@pytest.mark.parametrize("call", [_attend(), _evict(), _evict4(), _attend(valid=None, lse=None), _evict(valid=None, dst_weight=None),
                                  _evict4(sel_idx=torch.zeros(9, dtype=I32)), _attend(out=torch.zeros(5, 4, 64), valid=torch.ones(6, dtype=torch.uint8))])
def test_what_fits_reaches_the_library(call):
    with pytest.raises(pc.PackCacheError, match="pc_.*evict: invalid|pc_q4_attend: invalid") as e:            # which refuses a null context
        call()
    assert e.value.status == pc.PC_ERR_INVALID_ARG


def test_masses_and_weights_are_fp32():
    with pytest.raises(AssertionError, match="fp32"):
        pc.pc_accumulate(_Closed, torch.zeros(4), torch.zeros(4).double(), 1.0, 1.0, stream=0)
