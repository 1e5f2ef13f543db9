"""The paged 8-bit cache's argument checks, which need no GPU, and its reference."""
import ctypes as C
import os

import numpy as np
import pytest
import torch

import page_ref as ref
from paper_2603_22910_amd import binding as ek

FAKE = 0x100000  # non-null stand-in for a device pointer; never dereferenced on these paths


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(ek.LIB_PATH):
        from paper_2603_22910_amd import build
        build.build_library()
    return ek.load()


class Table:
    def __init__(self, **kw):
        self.c = ek.PageTableC(**{**dict(batch=2, max_pages=4, n_pages=8, table=FAKE, seq_len=FAKE, free_list=FAKE, n_free=FAKE), **kw})
        self.batch, self.n_pages, self.seq_len, self.n_free = self.c.batch, self.c.n_pages, FAKE, FAKE

    def as_c(self):
        return self.c


class Cache:
    def __init__(self, **kw):
        self.c = ek.PageCacheC(**{**{n: FAKE for n, _ in ek.PageCacheC._fields_}, **kw})

    def as_c(self, shape, t):
        return self.c


class Plan:
    def __init__(self, **kw):
        self.c = ek.PagePlanC(**{**dict(buf=FAKE, bytes=1 << 20, max_rows=10), **kw})
        self.max_rows = self.c.max_rows

    def as_c(self):
        return self.c


class Ws:
    def __init__(self, n, p=FAKE):
        self.n, self.p = n, p

    def numel(self): return self.n
    def element_size(self): return 1
    def data_ptr(self): return self.p


SHAPE = ek.make_shape(8, 2, 128, 0, "bf16")


def calls(shape=SHAPE, t=None, c=None, plan=None, ptr=FAKE, out=FAKE, ws=None, **kw):
    """Every entry point with these arguments: its name and status."""
    t, c, plan, ws = t or Table(), c or Cache(), plan or Plan(), ws or Ws(1)          # the workspace is too small: nothing is ever launched
    run = {
        "grow": lambda: ek.pages_grow(shape, t, ptr, plan, stream=0),
        "slots": lambda: ek.pages_slots(t, ptr, ptr, ptr, n_rows=5, stream=0),
        "release": lambda: ek.pages_release(t, ptr, stream=0),
        "append": lambda: ek.page_append(shape, t, c, plan, ptr, ptr, stream=0),
        "read": lambda: ek.page_read(shape, t, c, ptr, out, out, n_rows=5, stream=0),
        "decode": lambda: ek.page_decode_attn(shape, t, c, plan, ptr, out, None, ws, stream=0, **kw),
        "prefill": lambda: ek.page_prefill_attn(shape, t, c, plan, ptr, out, None, ws, stream=0, **kw),
    }
    return run


def codes(only, **kw):
    out = {}
    for name, f in calls(**kw).items():
        if name not in only:
            continue
        try:
            f()
            out[name] = ek.OK
        except ek.EchoKVError as e:
            out[name] = e.code
    return out


SHAPED, ATTN = ("grow", "append", "read", "decode", "prefill"), ("decode", "prefill")


@pytest.mark.parametrize("shape,want", [
    (ek.make_shape(8, 3, 128, 0, "bf16"), ek.ERR_SHAPE), (ek.make_shape(0, 1, 128, 0, "bf16"), ek.ERR_SHAPE),
    (ek.make_shape(8, 2, 96, 0, "bf16"), ek.ERR_UNSUPPORTED), (ek.make_shape(8, 2, 128, 0, "f32"), ek.ERR_UNSUPPORTED),
    (ek.make_shape(8, 2, 128, 0, "bf16", flags=ek.FLAG_UNFUSED), ek.ERR_UNSUPPORTED),
    (ek.make_shape(8, 2, 128, 0, "bf16", softmax_scale=float("nan")), ek.ERR_SHAPE)])
def test_shapes(shape, want):
    assert codes(SHAPED, shape=shape) == {n: want for n in SHAPED}
    assert ek.page_workspace_bytes(shape, 2, 10) == 0


@pytest.mark.parametrize("change,want", [
    (dict(batch=0), ek.ERR_SHAPE), (dict(max_pages=0), ek.ERR_SHAPE), (dict(n_pages=-1), ek.ERR_SHAPE), (dict(batch=4097), ek.ERR_UNSUPPORTED),
    (dict(n_pages=1 << 24), ek.ERR_UNSUPPORTED), (dict(max_pages=1 << 23), ek.ERR_UNSUPPORTED), (dict(table=None), ek.ERR_NULL),
    (dict(seq_len=None), ek.ERR_NULL), (dict(free_list=None), ek.ERR_NULL), (dict(n_free=None), ek.ERR_NULL)])
def test_tables(change, want):
    every = SHAPED + ("slots", "release")
    assert codes(every, t=Table(**change)) == {n: want for n in every}


@pytest.mark.parametrize("name", [n for n, _ in ek.PageCacheC._fields_])
def test_caches(name):
    names = ("append", "read", "decode", "prefill")
    assert codes(names, c=Cache(**{name: None})) == {n: ek.ERR_NULL for n in names}
    if "exp" not in name:
        assert codes(names, c=Cache(**{name: FAKE + 8})) == {n: ek.ERR_SHAPE for n in names}


@pytest.mark.parametrize("change,want", [(dict(buf=None), ek.ERR_NULL), (dict(max_rows=-1), ek.ERR_SHAPE), (dict(max_rows=(1 << 30) + 1), ek.ERR_SHAPE),
                                         (dict(max_rows=1 << 28), ek.ERR_UNSUPPORTED),
                                         (dict(bytes=64), ek.ERR_WORKSPACE), (dict(buf=FAKE + 4), ek.ERR_WORKSPACE)])
def test_plans(change, want):
    names = ("grow", "append", "decode", "prefill")
    assert codes(names, plan=Plan(**change)) == {n: want for n in names}


def test_rows_queries_outputs_and_workspaces():
    assert codes(SHAPED + ("slots", "release"), ptr=None) == {n: ek.ERR_NULL for n in SHAPED + ("slots", "release")}
    assert codes(("append",) + ATTN, ptr=FAKE + 2) == {n: ek.ERR_SHAPE for n in ("append",) + ATTN}
    assert codes(("read",) + ATTN, out=None) == {n: ek.ERR_NULL for n in ("read",) + ATTN}
    assert codes(("read",) + ATTN, out=FAKE + 2) == {n: ek.ERR_SHAPE for n in ("read",) + ATTN}
    for cap in (-1.0, float("inf"), float("nan"), 1e-31, 2e37):
        assert codes(ATTN, softcap=cap) == {n: ek.ERR_SHAPE for n in ATTN}
    assert codes(ATTN) == {n: ek.ERR_WORKSPACE for n in ATTN}
    need = ek.page_workspace_bytes(SHAPE, 2, 10)
    assert codes(("decode",), ws=Ws(need, FAKE + 8)) == {"decode": ek.ERR_WORKSPACE}
    assert ek.page_workspace_bytes(SHAPE, 0, 10) == 0 and ek.page_workspace_bytes(SHAPE, 4097, 10) == 0
    assert 0 < ek.page_workspace_bytes(SHAPE, 2, 0) <= need
    assert ek.page_plan_bytes(0) == 0 and ek.page_plan_bytes(4097) == 0 and ek.page_plan_bytes(4096) > 4096 * 4
    # no new rows at all: nothing to store, no queries
    assert codes(("append", "prefill"), plan=Plan(max_rows=0)) == {"append": ek.OK, "prefill": ek.OK}


def test_the_binding_checks_tensors():
    t = torch.zeros(4, 4, dtype=torch.int32)
    with pytest.raises(ValueError, match="not on a GPU"):
        ek.pages_release(Table(), t)
    with pytest.raises(TypeError, match="expected int32"):
        ek.pages_release(Table(), t.long())
    with pytest.raises(ValueError, match="not contiguous"):
        ek.pages_release(Table(), t.T[1:])


def test_views_follow_their_tensors():
    class T:                                                 # a tensor's address and shape
        def __init__(self, p, *shape): self.p, self.shape = p, shape
        def data_ptr(self): return self.p
    t = ek.PageTable(T(FAKE, 3, 7), T(FAKE + 64, 3), T(FAKE + 128, 9), T(FAKE + 192, 1))
    c = t.as_c()
    assert (c.batch, c.max_pages, c.n_pages, c.table, c.n_free) == (3, 7, 9, FAKE, FAKE + 192) and t.as_c() is c
    t.seq_len.p = FAKE + 256                                 # other storage behind the same tensor
    assert t.as_c() is not c and t.as_c().seq_len == FAKE + 256
    t.free_list = T(FAKE + 320, 11)
    assert t.as_c().n_pages == t.n_pages == 11 and t.as_c().free_list == FAKE + 320
    cache = ek.PageCache(*(T(FAKE + 64 * i, 9) for i in range(6)))
    a = cache.as_c(SHAPE, t)
    assert cache.as_c(SHAPE, t) is a and cache.as_c(ek.make_shape(8, 4, 128, 0, "bf16"), t) is not a


def test_views_are_checked_again_when_another_gpu_is_the_current_one(monkeypatch):
    class T:
        shape = (9,)
        def data_ptr(self): return FAKE
    t = ek.PageTable(type("T2", (T,), dict(shape=(3, 7)))(), T(), T(), T())
    monkeypatch.setitem(ek._DTYPES, "device", lambda: 0)
    first = t.as_c()
    assert t.as_c() is first
    monkeypatch.setitem(ek._DTYPES, "device", lambda: 1)
    assert t.as_c() is not first


@pytest.mark.parametrize("scale", [1e-11, 1e-40, 1e11])
def test_scales_of_scores_that_leave_the_range(scale):
    shape = ek.make_shape(8, 2, 128, 0, "bf16", softmax_scale=scale)
    assert codes(SHAPED, shape=shape) == {n: ek.ERR_SHAPE for n in SHAPED}
    assert ek.page_workspace_bytes(shape, 2, 10) == 0


@pytest.mark.parametrize("cap", [1e-21, 1e21, 1e37])
def test_caps_that_leave_the_range(cap):
    assert codes(ATTN, softcap=cap) == {n: ek.ERR_SHAPE for n in ATTN}


def test_reference_rounding_and_scales():
    codes = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double()
    codes = torch.sort(codes[torch.isfinite(codes)]).values
    assert torch.equal(ref.e4m3(codes), codes)
    mid = (codes[1:] + codes[:-1]) / 2                       # ties go to the neighbour whose last bit is 0, as torch's cast does it
    assert torch.equal(ref.e4m3(mid), mid.float().to(torch.float8_e4m3fn).double())
    x = torch.zeros(128, 1, 64, dtype=torch.bfloat16)
    x[0, 0, 0], x[1, 0, 1] = 448.0, 1.0
    assert ref.held(x)[1, 0, 1] == 1.0 and ref.held(x)[0, 0, 0] == 448.0
    x[0, 0, 0] = 450.0
    assert ref.held(x)[0, 0, 0] == 448.0                     # 450 / 2 = 225 between 224 and 240
