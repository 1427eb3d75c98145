"""The paged cache: what its calls refuse, without a GPU.  Types and lengths are looked at before the library is called, so a context that is closed is enough to see that; the library's own checks run over a
CUDA runtime that runs nothing."""
from __future__ import annotations

import pytest
import torch

from paper_2601_04359_b200 import binding as pc
from tests.host_runtime import rt, _library      # noqa: F401  (fixtures)

I32 = torch.int32


class _Closed:
    handle, device = None, -1
    sizes = (4, 2, 64, torch.float32)


class _Work:
    handle, ctx = None, _Closed


def _pages(n=3, page=16, heads=2, dtype=torch.float32):
    return pc.Pages(torch.zeros(n, page, heads, 64, dtype=dtype), torch.zeros(n, page, heads, 64, dtype=dtype))


def _batch(**kw):
    a = dict(table=torch.zeros(2, 3, dtype=I32), length=torch.ones(2, dtype=I32), row_start=torch.tensor([0, 1, 2], dtype=I32), max_rows=1, prefix=None, n_prefix=0)
    return pc.Batch(**{**a, **kw})


def _append(pages=None, batch=None, **kw):
    a = {"k": torch.zeros(2, 2, 64), "v": torch.zeros(2, 2, 64), "pos": torch.zeros(2, 4, dtype=I32), **kw}
    return lambda: pc.pc_paged_append(_Closed, pages or _pages(), batch or _batch(), stream=0, **a)


def _attend(pages=None, batch=None, **kw):
    a = {"q": torch.zeros(2, 4, 64), "q_pos": torch.zeros(2, 4, dtype=I32), "out": torch.zeros(2, 4, 64), "lse": torch.zeros(2, 4), **kw}
    return lambda: pc.pc_paged_attend(_Work, pages or _pages(), batch or _batch(), stream=0, **a)


REFUSED = {
    "k in bf16": _append(k=torch.zeros(2, 2, 64, dtype=torch.bfloat16)),
    "k of other heads": _append(k=torch.zeros(2, 3, 64)),
    "v shorter": _append(v=torch.zeros(1, 2, 64)),
    "pos in 64 bits": _append(pos=torch.zeros(2, 4, dtype=torch.int64)),
    "pos shorter": _append(pos=torch.zeros(1, 4, dtype=I32)),
    "pages in bf16": _append(pages=_pages(dtype=torch.bfloat16)),
    "pages of other heads": _append(pages=_pages(heads=3)),
    "values of fewer pages": _append(pages=pc.Pages(torch.zeros(3, 16, 2, 64), torch.zeros(2, 16, 2, 64))),
    "no pages": _append(pages=pc.Pages(None, None)),
    "table in 64 bits": _append(batch=_batch(table=torch.zeros(2, 3, dtype=torch.int64))),
    "table of fewer sequences": _append(batch=_batch(table=torch.zeros(1, 3, dtype=I32))),
    "no table": _append(batch=_batch(table=None)),
    "length in 64 bits": _append(batch=_batch(length=torch.ones(2, dtype=torch.int64))),
    "row starts without an end": _append(batch=_batch(row_start=torch.tensor([0, 1], dtype=I32))),
    "prefix shorter than its tokens": _attend(batch=_batch(prefix=torch.zeros(1, dtype=I32), n_prefix=17)),
    "too many sequences": _attend(batch=_batch(table=torch.zeros(600, 1, dtype=I32), length=torch.zeros(600, dtype=I32), row_start=torch.zeros(601, dtype=I32))),
    "q of other heads": _attend(q=torch.zeros(2, 3, 64)),
    "q in bf16": _attend(q=torch.zeros(2, 4, 64, dtype=torch.bfloat16)),
    "q_pos shorter": _attend(q_pos=torch.zeros(1, 4, dtype=I32)),
    "out shorter": _attend(out=torch.zeros(1, 4, 64)),
    "out in bf16": _attend(out=torch.zeros(2, 4, 64, dtype=torch.bfloat16)),
    "lse in 64 bits": _attend(lse=torch.zeros(2, 4, dtype=torch.float64)),
    "lse shorter": _attend(lse=torch.zeros(1, 4)),
    "no context": _append(),
    "no workspace": _attend(),
}


@pytest.mark.parametrize("case", list(REFUSED))
def test_refused(case):
    with pytest.raises(pc.PackCacheError) as e:
        REFUSED[case]()
    assert e.value.status == pc.PC_ERR_INVALID_ARG


@pytest.mark.parametrize("call", [_append(k=torch.zeros(2, 2, 128)[..., ::2]), _attend(q=torch.zeros(4, 2, 64).transpose(0, 1))])
def test_tensors_have_to_be_contiguous(call):
    with pytest.raises(AssertionError):
        call()


class _Case:
    """The C entry points over the runtime that runs nothing; fields of the two structs and the arguments can be given by name."""

    def __init__(self, rt, max_q=8):
        self.ctx = pc.Context(24, 8, 128, pc.PC_BF16, 10000.0, (64, 64, 64), max_q, 1)
        self.work = pc.PagedWork(self.ctx)
        rt.open += [self.ctx, self.work]
        self.room = torch.zeros(1 << 16, dtype=torch.uint8)
        self.at = (self.room.data_ptr() + 15) // 16 * 16

    def call(self, name, **kw):
        at = self.at
        pages = dict(k=at, v=at, n_pages=4, page_tokens=16)
        batch = dict(table=at, length=at, row_start=at, prefix=None, n_seqs=2, max_pages=3, n_prefix=0, max_rows=1)
        args = dict(a=at, b=at, pos=at, n_rows=2, out=at, lse=None)
        for k, v in kw.items():
            where = next(d for d in (pages, batch, args) if k in d)
            where[k] = v
        p, b = pc.pc_pages(**pages), pc.pc_batch(**batch)
        if name == "append":
            return pc.load().pc_paged_append(self.ctx.handle, p, b, args["a"], args["b"], args["pos"], args["n_rows"], None)
        return pc.load().pc_paged_attend(self.work.handle, p, b, args["a"], args["pos"], args["n_rows"], 1, args["out"], args["lse"], None)


def _launches(rt):
    return [line for line in rt.log() if line.startswith("launch")]


BOTH, ATTEND, APPEND = ("append", "attend"), ("attend",), ("append",)
CHECKS = {
    "page of 8": (BOTH, dict(page_tokens=8), pc.PC_ERR_UNSUPPORTED),
    "page of 24": (BOTH, dict(page_tokens=24), pc.PC_ERR_UNSUPPORTED),
    "page of 256": (BOTH, dict(page_tokens=256), pc.PC_ERR_UNSUPPORTED),
    "no keys": (BOTH, dict(k=None), pc.PC_ERR_INVALID_ARG),
    "no values": (BOTH, dict(v=None), pc.PC_ERR_INVALID_ARG),
    "no pages": (BOTH, dict(n_pages=0), pc.PC_ERR_INVALID_ARG),
    "2^31 tokens": (BOTH, dict(n_pages=1 << 24, page_tokens=128), pc.PC_ERR_CAPACITY),
    "no table": (BOTH, dict(table=None), pc.PC_ERR_INVALID_ARG),
    "no lengths": (BOTH, dict(length=None), pc.PC_ERR_INVALID_ARG),
    "no row starts": (BOTH, dict(row_start=None), pc.PC_ERR_INVALID_ARG),
    "prefix without pages": (BOTH, dict(n_prefix=5), pc.PC_ERR_INVALID_ARG),
    "negative prefix": (BOTH, dict(n_prefix=-1), pc.PC_ERR_INVALID_ARG),
    "negative rows": (BOTH, dict(n_rows=-1), pc.PC_ERR_INVALID_ARG),
    "negative most rows": (BOTH, dict(max_rows=-1), pc.PC_ERR_INVALID_ARG),
    "negative sequences": (BOTH, dict(n_seqs=-1), pc.PC_ERR_INVALID_ARG),
    "513 sequences": (BOTH, dict(n_seqs=513), pc.PC_ERR_CAPACITY),
    "more rows than max_q": (BOTH, dict(n_rows=9), pc.PC_ERR_CAPACITY),
    "a table of 2^31 tokens": (BOTH, dict(max_pages=1 << 27), pc.PC_ERR_CAPACITY),
    "nowhere to append": (APPEND, dict(max_pages=0), pc.PC_ERR_INVALID_ARG),
    "no queries or keys": (BOTH, dict(a=None), pc.PC_ERR_INVALID_ARG),
    "no new values": (APPEND, dict(b=None), pc.PC_ERR_INVALID_ARG),
    "no positions": (BOTH, dict(pos=None), pc.PC_ERR_INVALID_ARG),
    "no output": (ATTEND, dict(out=None), pc.PC_ERR_INVALID_ARG),
}


@pytest.mark.parametrize("case", list(CHECKS))
def test_the_librarys_own_checks(rt, case):      # noqa: F811
    names, kw, status = CHECKS[case]
    c = _Case(rt)
    for name in names:
        assert c.call(name, **kw) == status
    assert not _launches(rt)


def test_misaligned_memory_and_another_device(rt):      # noqa: F811
    c = _Case(rt)
    for field in ("k", "v", "a", "pos"):
        for name in BOTH:
            assert c.call(name, **{field: c.at + 8}) == pc.PC_ERR_INVALID_ARG
    for field in ("table", "length", "row_start"):
        for name in BOTH:
            assert c.call(name, **{field: c.at + 2}) == pc.PC_ERR_INVALID_ARG
    assert c.call("attend", out=c.at + 8) == c.call("attend", lse=c.at + 4) == pc.PC_ERR_INVALID_ARG
    rt.device(1)
    assert c.call("attend") == c.call("append") == pc.PC_ERR_INVALID_ARG
    rt.device(0)
    assert not _launches(rt)


def test_nothing_to_do_launches_nothing(rt):      # noqa: F811
    c = _Case(rt)
    for name in BOTH:
        assert c.call(name, n_seqs=0, table=None, length=None) == pc.PC_OK
        assert c.call(name, n_rows=0) == pc.PC_OK
    assert c.call("attend", max_rows=0) == pc.PC_OK
    assert not _launches(rt)
