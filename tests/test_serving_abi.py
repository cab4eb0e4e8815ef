"""Refusals of the serving-step entry points, on the host before anything is launched, and the rotary plan."""
import ctypes as C
import math

import pytest
import torch

from paper_2607_20538_amd import codec as cg

BU = cg.Codec(cg.BLOCK_UNIFORM, 4, 32)
PTR = 0x10000


def _view(L=1, B=1, H=2, T=16, d=64, dtype=cg.DTYPE_BF16, ptr=PTR, strides=None):
    return cg.KvView(ptr, dtype, L, B, H, T, d, *(strides or (B * H * T * d, H * T * d, T * d, d)))


def _cache(L=1, B=4, H=2, T_cap=64, d=64, codes=0x20000, side=0x30000):
    return cg.CacheStruct(codes, side, None, L, B, H, T_cap, d, 0)


def _pool(free=PTR, count=PTR, n=8):
    return cg.PagePoolStruct(free, count, n)


# ------------------------------------------------------------------------------------------
# tables
# ------------------------------------------------------------------------------------------

def _map(held=PTR, add=PTR, B=2, pool=None, pages=PTR, max_pages=4, P=64, N=8, cu=PTR, lens=PTR, pos=PTR, slots=PTR, err=None):
    p = pool or _pool()
    return cg.lib().kv_page_map(held, add, B, C.byref(p), pages, max_pages, P, N, cu, lens, pos, slots, err, None)


@pytest.mark.parametrize("kw,status", [
    (dict(held=None), cg.CG_ERR_ARG), (dict(add=None), cg.CG_ERR_ARG), (dict(pages=None), cg.CG_ERR_ARG),
    (dict(cu=None), cg.CG_ERR_ARG), (dict(lens=None), cg.CG_ERR_ARG), (dict(pos=None), cg.CG_ERR_ARG),
    (dict(slots=None), cg.CG_ERR_ARG), (dict(B=0), cg.CG_ERR_ARG), (dict(N=-1), cg.CG_ERR_ARG),
    (dict(max_pages=0), cg.CG_ERR_ARG), (dict(pool=_pool(free=None)), cg.CG_ERR_ARG),
    (dict(pool=_pool(count=None)), cg.CG_ERR_ARG), (dict(pool=_pool(n=0)), cg.CG_ERR_ARG),
    (dict(P=0), cg.CG_ERR_SHAPE), (dict(P=65), cg.CG_ERR_SHAPE), (dict(held=PTR + 2), cg.CG_ERR_ALIGN),
    (dict(slots=PTR + 1), cg.CG_ERR_ALIGN), (dict(err=PTR + 2), cg.CG_ERR_ALIGN), (dict(pages=PTR + 2), cg.CG_ERR_ALIGN),
    (dict(pool=_pool(n=2 ** 25)), cg.CG_ERR_CAPACITY), (dict(max_pages=2 ** 25), cg.CG_ERR_CAPACITY),
])
def test_page_map_refuses(kw, status):
    assert _map(**kw) == status


def test_page_release_refuses():
    p = _pool()
    call = lambda lens=PTR, done=PTR, B=2, pool=p, P=64: cg.lib().kv_page_release(  # noqa: E731
        lens, done, B, C.byref(pool), PTR, 4, P, None, None)
    assert call(lens=None) == cg.CG_ERR_ARG and call(done=None) == cg.CG_ERR_ARG and call(B=0) == cg.CG_ERR_ARG
    assert call(P=63) == cg.CG_ERR_SHAPE and call(done=PTR + 2) == cg.CG_ERR_ALIGN
    assert call(pool=_pool(n=2 ** 26)) == cg.CG_ERR_CAPACITY


# ------------------------------------------------------------------------------------------
# rotary positions
# ------------------------------------------------------------------------------------------

@pytest.mark.parametrize("kw", [
    dict(d_rot=0), dict(d_rot=7), dict(d_rot=258), dict(layout=2), dict(scaling=3), dict(scaling=-1), dict(base=0.0),
    dict(base=-5.0), dict(base=math.inf), dict(base=math.nan), dict(amplitude=math.inf), dict(amplitude=1e300),
    dict(scaling=cg.ROPE_LINEAR, factor=0.0), dict(scaling=cg.ROPE_LINEAR, factor=math.nan),
    dict(scaling=cg.ROPE_RAMP, factor=2.0, train_len=0), dict(scaling=cg.ROPE_RAMP, factor=2.0, train_len=9, low=4.0, high=4.0),
    dict(scaling=cg.ROPE_RAMP, factor=2.0, train_len=9, low=math.nan),
])
def test_rope_make_refuses(kw):
    with pytest.raises(cg.CodecError) as e:
        cg.rope_make(**{**dict(d_rot=64), **kw})
    assert e.value.status == cg.CG_ERR_ARG


def test_rope_plan_holds_turns_per_position():
    plan = cg.rope_make(128, cg.ROPE_PAIRS, base=500000.0, amplitude=0.5)
    assert plan.d_rot == 128 and plan.layout == cg.ROPE_PAIRS and plan.amplitude == 0.5
    for i in range(64):
        turns = 500000.0 ** (-2 * i / 128) / (2 * math.pi)
        # two binary64 roundings of the power, one of the quotient
        assert abs(plan.step[i] / 2 ** 64 - turns) <= 4 * 2.0 ** -53 * turns + 2.0 ** -64
    lin, none = cg.rope_make(8, scaling=cg.ROPE_LINEAR, factor=8.0), cg.rope_make(8)
    assert all(abs(a * 8 - b) <= 2 ** 13 for a, b in zip(lin.step[:4], none.step[:4]))
    ramp = cg.rope_make(8, scaling=cg.ROPE_RAMP, factor=8.0, low=1.0, high=2.0, train_len=100)
    # pairs make 15.9, 1.59, 0.16, 0.016 turns over 100 positions: kept, blended, divided, divided
    assert ramp.step[0] == none.step[0] and ramp.step[2] == lin.step[2] and lin.step[1] < ramp.step[1] < none.step[1]
    # a base below one: whole turns per position are none
    up = cg.rope_make(4, base=1e-4)
    assert abs(up.step[1] / 2 ** 64 - (100 / (2 * math.pi)) % 1) <= 1e-13


def _rope(x0=None, y0=None, x1=None, y1=None, pos=PTR, rot=64, plan=None):
    plan = plan or cg.rope_make(rot)
    x0 = x0 or _view()
    y0 = y0 or _view()
    b = lambda v: None if v is None else C.byref(v)  # noqa: E731
    return cg.lib().kv_rope(C.byref(plan), b(x0), b(y0), b(x1), b(y1), pos, 0, None)


@pytest.mark.parametrize("kw,status", [
    (dict(x1=_view()), cg.CG_ERR_ARG), (dict(y1=_view()), cg.CG_ERR_ARG), (dict(pos=None), cg.CG_ERR_ARG),
    (dict(pos=PTR + 2), cg.CG_ERR_ALIGN), (dict(rot=66), cg.CG_ERR_SHAPE), (dict(y0=_view(T=15)), cg.CG_ERR_SHAPE),
    (dict(y0=_view(H=1)), cg.CG_ERR_SHAPE), (dict(y0=_view(dtype=cg.DTYPE_F32)), cg.CG_ERR_SHAPE),
    (dict(x1=_view(H=4), y1=_view(H=3)), cg.CG_ERR_SHAPE), (dict(x1=_view(T=3), y1=_view(T=3)), cg.CG_ERR_SHAPE),
    (dict(x0=_view(ptr=PTR + 8)), cg.CG_ERR_ALIGN), (dict(x0=_view(strides=(4, 4, 4, 68))), cg.CG_ERR_ALIGN),
    (dict(x0=_view(ptr=None)), cg.CG_ERR_ARG), (dict(x0=_view(dtype=7)), cg.CG_ERR_ARG),
    (dict(x0=_view(strides=(-64, 64, 64, 64))), cg.CG_ERR_ARG), (dict(x0=_view(d=68), y0=_view(d=68)), cg.CG_ERR_ALIGN),
    (dict(x0=_view(d=264), y0=_view(d=264)), cg.CG_ERR_UNSUPPORTED), (dict(x0=_view(H=0), y0=_view(H=0)), cg.CG_ERR_SHAPE),
    (dict(x0=_view(T=2 ** 26 + 1, strides=(0, 0, 0, 64)), y0=_view(T=2 ** 26 + 1, strides=(0, 0, 0, 64))), cg.CG_ERR_CAPACITY),
    (dict(x0=_view(H=70000, strides=(0, 0, 0, 64)), y0=_view(H=70000, strides=(0, 0, 0, 64))), cg.CG_ERR_CAPACITY),
])
def test_rope_refuses(kw, status):
    assert _rope(**kw) == status


def test_rope_of_nothing():
    assert _rope(x0=_view(T=0, ptr=None), y0=_view(T=0, ptr=None), pos=None) == cg.CG_OK


# ------------------------------------------------------------------------------------------
# packed tokens
# ------------------------------------------------------------------------------------------

def _append(k=None, v=None, slots=PTR, shp=None, codec=BU, kc=None, vc=None, l0=0, l1=1, gdev=0x50000, err=None):
    cs = codec.struct()
    k, v, kc, vc = k or _view(), v or _view(), kc or _cache(), vc or _cache()
    return cg.lib().kv_append_slots(l0, l1, C.byref(k), C.byref(v), slots, gdev, shp or cg.shape(1, 2, 64, 16), C.byref(cs),
                                    C.byref(kc), C.byref(vc), err, None)


@pytest.mark.parametrize("kw,status", [
    (dict(slots=None), cg.CG_ERR_ARG), (dict(slots=PTR + 2), cg.CG_ERR_ALIGN), (dict(gdev=None), cg.CG_ERR_ARG),
    (dict(gdev=PTR + 4), cg.CG_ERR_ALIGN), (dict(l1=2), cg.CG_ERR_ARG), (dict(l0=1), cg.CG_ERR_ARG),
    (dict(k=_view(B=2), v=_view(B=2)), cg.CG_ERR_SHAPE), (dict(v=_view(T=15)), cg.CG_ERR_SHAPE),
    (dict(k=_view(H=3)), cg.CG_ERR_SHAPE), (dict(kc=_cache(T_cap=32), vc=_cache(T_cap=32)), cg.CG_ERR_SHAPE),
    (dict(vc=_cache(T_cap=128)), cg.CG_ERR_SHAPE), (dict(vc=_cache(B=5)), cg.CG_ERR_SHAPE),
    (dict(kc=_cache(side=None)), cg.CG_ERR_ARG), (dict(kc=_cache(codes=PTR + 8)), cg.CG_ERR_ALIGN),
    (dict(codec=cg.Codec(cg.KIVI, 4, 32, 32, 32, 32)), cg.CG_ERR_ARG),
    (dict(codec=cg.Codec(cg.ZFP, 4)), cg.CG_ERR_UNSUPPORTED),
    (dict(codec=cg.Codec(cg.BLOCK_UNIFORM, 5, 32)), cg.CG_ERR_UNSUPPORTED),
    (dict(kc=_cache(B=2 ** 25, T_cap=64), vc=_cache(B=2 ** 25, T_cap=64)), cg.CG_ERR_CAPACITY),
    (dict(err=PTR + 1), cg.CG_ERR_ALIGN), (dict(k=_view(T=0, ptr=None), v=_view(T=0, ptr=None), slots=None), cg.CG_OK),
])
def test_append_slots_refuses(kw, status):
    assert _append(**kw) == status


def _attend(q=None, out=None, cu=PTR, B=2, max_q=8, kc=None, vc=None, pages=PTR, max_pages=4, P=64, shp=None, codec=BU, lens=PTR,
            scale=0.1, window=0, sinks=0, ws=PTR, l0=0, l1=1, gdev=0x50000, err=None):
    cs = codec.struct()
    q, out, kc, vc = q or _view(H=4), out or _view(H=4), kc or _cache(), vc or _cache()
    pt = cg.PageTable(pages, max_pages, P)
    return cg.lib().kv_attend_chunk_paged(l0, l1, C.byref(q), cu, B, max_q, C.byref(kc), C.byref(vc), C.byref(pt), gdev,
                                          shp or cg.shape(1, 2, 64, 16), C.byref(cs), lens, scale, window, sinks, C.byref(out),
                                          ws, err, None)


@pytest.mark.parametrize("kw,status", [
    (dict(cu=None), cg.CG_ERR_ARG), (dict(lens=None), cg.CG_ERR_ARG), (dict(pages=None), cg.CG_ERR_ARG),
    (dict(cu=PTR + 2), cg.CG_ERR_ALIGN), (dict(lens=PTR + 2), cg.CG_ERR_ALIGN), (dict(pages=PTR + 2), cg.CG_ERR_ALIGN),
    (dict(err=PTR + 2), cg.CG_ERR_ALIGN), (dict(gdev=None), cg.CG_ERR_ARG), (dict(B=0), cg.CG_ERR_ARG),
    (dict(max_q=0), cg.CG_ERR_ARG), (dict(window=-1), cg.CG_ERR_ARG), (dict(sinks=-1), cg.CG_ERR_ARG),
    (dict(scale=math.nan), cg.CG_ERR_ARG), (dict(scale=math.inf), cg.CG_ERR_ARG), (dict(l1=2), cg.CG_ERR_ARG),
    (dict(q=_view(H=3), out=_view(H=3)), cg.CG_ERR_SHAPE), (dict(q=_view(H=1), out=_view(H=1)), cg.CG_ERR_SHAPE),
    (dict(q=_view(H=4, B=2), out=_view(H=4, B=2)), cg.CG_ERR_SHAPE), (dict(out=_view(H=4, T=15)), cg.CG_ERR_SHAPE),
    (dict(out=_view(H=2)), cg.CG_ERR_SHAPE), (dict(q=_view(H=4, d=72)), cg.CG_ERR_SHAPE),
    (dict(q=_view(H=4, ptr=PTR + 8)), cg.CG_ERR_ALIGN), (dict(P=128), cg.CG_ERR_SHAPE), (dict(P=32), cg.CG_ERR_SHAPE),
    (dict(vc=_cache(T_cap=128)), cg.CG_ERR_SHAPE), (dict(codec=cg.Codec(cg.ZFP, 4)), cg.CG_ERR_UNSUPPORTED),
    (dict(codec=cg.Codec(cg.BLOCK_UNIFORM, 4, 32, block_t=16)), cg.CG_ERR_ARG),
    (dict(max_pages=2 ** 25), cg.CG_ERR_CAPACITY), (dict(max_pages=0), cg.CG_ERR_ARG),
    (dict(max_pages=200, max_q=1, ws=None), cg.CG_ERR_ARG), (dict(max_pages=200, max_q=1, ws=PTR + 8), cg.CG_ERR_ALIGN),
    (dict(q=_view(H=4, T=0, ptr=None), out=_view(H=4, T=0, ptr=None)), cg.CG_OK),
])
def test_attend_chunk_refuses(kw, status):
    assert _attend(**kw) == status


def test_chunk_workspace():
    shp = cg.shape(1, 8, 128, 128)
    n = lambda *a: cg.attend_chunk_workspace_bytes(shp, *a)  # noqa: E731
    assert n(1, 4096, 1, 4096, 32, 400, 64) == 0                 # enough tiles: no splits
    assert n(1, 1, 1, 1, 32, 400, 64) > 0                        # one token over a long row
    assert n(1, 1, 1, 1, 32, 400, 64, 64, 4) == 0                # a short window
    assert n(0, 1, 1, 1, 32, 400, 64) == 0 and n(1, 1, 1, 1, 31, 400, 64) == 0 and n(1, 1, 1, 1, 32, 400, 63) == 0


def test_binding_refuses_host_tensors_and_other_types():
    t = torch.zeros((1, 1, 2, 4, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        cg.kv_rope(cg.rope_make(64), t, t, torch.zeros((1, 4), dtype=torch.int32))
    with pytest.raises(ValueError):
        cg._int32("f", 4, pos=torch.zeros(4, dtype=torch.int64))
    with pytest.raises(ValueError):
        cg._int32("f", 4, pos=torch.zeros(5, dtype=torch.int32))
    with pytest.raises(ValueError):
        cg._int32("f", None, pages=torch.zeros((4, 4), dtype=torch.int32).t())


@pytest.mark.parametrize("strides", [(0, 0, 0, 64), (2048, 2048, 1024, 0), (2048, 2048, 0, 64), (2048, 2048, 64, 64),
                                     (2048, 2048, 960, 64), (2048, 2048, 32, 128)])
def test_outputs_that_overlap_are_refused(strides):
    assert _rope(y0=_view(strides=strides)) == cg.CG_ERR_ARG
    assert _rope(x1=_view(), y1=_view(strides=strides)) == cg.CG_ERR_ARG
    assert _attend(q=_view(), out=_view(strides=strides)) == cg.CG_ERR_ARG


def test_append_slots_of_too_many_tokens():
    v = _view(T=2 ** 31 - 32, strides=(0, 0, 0, 0))
    assert _append(k=v, v=v) == cg.CG_ERR_CAPACITY


def test_attend_chunk_of_the_longest_tables():
    top = (2 ** 31 - 2 ** 16) // 64
    assert _attend(max_pages=top + 1) == cg.CG_ERR_CAPACITY
    assert _attend(max_pages=top, max_q=1, ws=None) == cg.CG_ERR_ARG
    shp = cg.shape(1, 2, 64, 16)
    assert cg.attend_chunk_workspace_bytes(shp, 1, 4, 1, 4, 4, top, 64) > 0
    assert cg.attend_chunk_workspace_bytes(shp, 1, 4, 1, 4, 4, top + 1, 64) == 0
