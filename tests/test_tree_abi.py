"""Refusals of the tree step's entry points, on the host before anything is launched."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from paper_2607_20538_amd import codec as cg

from test_serving_abi import BU, PTR, _cache, _pool, _view

import _tree as T


def _map(parent=PTR, cu=PTR, lens=PTR, B=2, N=8, words=1, pos=PTR, mask=PTR, err=None):
    return cg.lib().kv_tree_map(parent, cu, lens, B, N, words, pos, mask, err, None)


@pytest.mark.parametrize("kw,status", [
    (dict(parent=None), cg.CG_ERR_ARG), (dict(cu=None), cg.CG_ERR_ARG), (dict(lens=None), cg.CG_ERR_ARG),
    (dict(pos=None), cg.CG_ERR_ARG), (dict(mask=None), cg.CG_ERR_ARG), (dict(B=0), cg.CG_ERR_ARG),
    (dict(B=2 ** 31 - 1), cg.CG_ERR_ARG), (dict(N=-1), cg.CG_ERR_ARG), (dict(words=0), cg.CG_ERR_ARG),
    (dict(parent=PTR + 2), cg.CG_ERR_ALIGN), (dict(cu=PTR + 2), cg.CG_ERR_ALIGN), (dict(lens=PTR + 1), cg.CG_ERR_ALIGN),
    (dict(pos=PTR + 2), cg.CG_ERR_ALIGN), (dict(mask=PTR + 4), cg.CG_ERR_ALIGN), (dict(err=PTR + 2), cg.CG_ERR_ALIGN),
])
def test_tree_map_refuses(kw, status):
    assert _map(**kw) == status


def _accept(parent=PTR, cu=PTR, draft=PTR, target=PTR, head=None, B=2, N=8, path=PTR, kept=PTR, nxt=PTR, err=None):
    return cg.lib().kv_tree_accept(parent, cu, draft, target, head, B, N, path, kept, nxt, err, None)


@pytest.mark.parametrize("kw,status", [
    (dict(parent=None), cg.CG_ERR_ARG), (dict(cu=None), cg.CG_ERR_ARG), (dict(draft=None), cg.CG_ERR_ARG),
    (dict(target=None), cg.CG_ERR_ARG), (dict(path=None), cg.CG_ERR_ARG), (dict(kept=None), cg.CG_ERR_ARG),
    (dict(nxt=None), cg.CG_ERR_ARG), (dict(B=0), cg.CG_ERR_ARG), (dict(N=-1), cg.CG_ERR_ARG),
    (dict(head=PTR + 2), cg.CG_ERR_ALIGN), (dict(draft=PTR + 2), cg.CG_ERR_ALIGN), (dict(path=PTR + 2), cg.CG_ERR_ALIGN),
    (dict(kept=PTR + 2), cg.CG_ERR_ALIGN), (dict(nxt=PTR + 2), cg.CG_ERR_ALIGN), (dict(err=PTR + 2), cg.CG_ERR_ALIGN),
])
def test_tree_accept_refuses(kw, status):
    assert _accept(**kw) == status


def _keep(path=PTR, kept=PTR, cu=PTR, lens=PTR, B=2, N=8, pages=PTR, max_pages=4, P=64, shp=None, codec=BU, kc=None, vc=None,
          held=2 * PTR, l0=0, l1=1, err=None):
    cs, pt = codec.struct(), cg.PageTable(pages, max_pages, P)
    kc, vc = kc or _cache(), vc or _cache()
    return cg.lib().kv_tree_keep(l0, l1, path, kept, cu, lens, B, N, C.byref(pt), shp or cg.shape(1, 2, 64, 64), C.byref(cs),
                                 C.byref(kc), C.byref(vc), held, err, None)


@pytest.mark.parametrize("kw,status", [
    (dict(path=None), cg.CG_ERR_ARG), (dict(kept=None), cg.CG_ERR_ARG), (dict(cu=None), cg.CG_ERR_ARG),
    (dict(lens=None), cg.CG_ERR_ARG), (dict(held=None), cg.CG_ERR_ARG), (dict(held=PTR), cg.CG_ERR_ARG),
    (dict(pages=None), cg.CG_ERR_ARG), (dict(B=0), cg.CG_ERR_ARG), (dict(N=-1), cg.CG_ERR_ARG),
    (dict(l0=1), cg.CG_ERR_ARG), (dict(l1=2), cg.CG_ERR_ARG), (dict(l0=-1), cg.CG_ERR_ARG),
    (dict(path=PTR + 2), cg.CG_ERR_ALIGN), (dict(held=2 * PTR + 2), cg.CG_ERR_ALIGN), (dict(pages=PTR + 2), cg.CG_ERR_ALIGN),
    (dict(err=PTR + 2), cg.CG_ERR_ALIGN), (dict(P=128), cg.CG_ERR_SHAPE), (dict(vc=_cache(T_cap=128)), cg.CG_ERR_SHAPE),
    (dict(kc=_cache(T_cap=32), vc=_cache(T_cap=32)), cg.CG_ERR_SHAPE), (dict(kc=_cache(H=3)), cg.CG_ERR_SHAPE),
    (dict(codec=cg.Codec(cg.ZFP, 4)), cg.CG_ERR_UNSUPPORTED), (dict(kc=_cache(codes=PTR + 8)), cg.CG_ERR_ALIGN),
    (dict(kc=_cache(B=2 ** 25), vc=_cache(B=2 ** 25)), cg.CG_ERR_CAPACITY), (dict(max_pages=2 ** 25), cg.CG_ERR_CAPACITY),
    (dict(B=2 ** 30), cg.CG_ERR_CAPACITY),
])
def test_tree_keep_refuses(kw, status):
    assert _keep(**kw) == status


def test_page_trim_refuses():
    p = _pool()
    call = lambda lens=PTR, keep=PTR, B=2, pool=p, P=64: cg.lib().kv_page_trim(  # noqa: E731
        lens, keep, B, C.byref(pool), PTR, 4, P, None, None)
    assert call(lens=None) == cg.CG_ERR_ARG and call(keep=None) == cg.CG_ERR_ARG and call(B=0) == cg.CG_ERR_ARG
    assert call(P=63) == cg.CG_ERR_SHAPE and call(keep=PTR + 2) == cg.CG_ERR_ALIGN
    assert call(pool=_pool(n=2 ** 26)) == cg.CG_ERR_CAPACITY


def _append(k=None, v=None, q=None, qo=None, pos=PTR, slots=PTR, plan=None, rot=64, shp=None, codec=BU, kc=None, vc=None, l0=0,
            l1=1, gdev=0x50000, err=None, no_plan=False):
    cs = codec.struct()
    plan = plan or cg.rope_make(rot)
    k, v, kc, vc = k or _view(), v or _view(), kc or _cache(), vc or _cache()
    b = lambda x: None if x is None else C.byref(x)  # noqa: E731
    return cg.lib().kv_append_rope(l0, l1, None if no_plan else C.byref(plan), C.byref(k), C.byref(v), b(q), b(qo), pos, slots, gdev,
                                   shp or cg.shape(1, 2, 64, 16), C.byref(cs), C.byref(kc), C.byref(vc), err, None)


def _bad_plan():
    p = cg.rope_make(64)
    p.layout = 5
    return p


@pytest.mark.parametrize("kw,status", [
    (dict(slots=None), cg.CG_ERR_ARG), (dict(pos=None), cg.CG_ERR_ARG), (dict(no_plan=True), cg.CG_ERR_ARG),
    (dict(slots=PTR + 2), cg.CG_ERR_ALIGN), (dict(pos=PTR + 2), cg.CG_ERR_ALIGN), (dict(err=PTR + 1), cg.CG_ERR_ALIGN),
    (dict(gdev=None), cg.CG_ERR_ARG), (dict(gdev=PTR + 4), cg.CG_ERR_ALIGN), (dict(l1=2), cg.CG_ERR_ARG), (dict(l0=1), cg.CG_ERR_ARG),
    (dict(q=_view(H=4)), cg.CG_ERR_ARG), (dict(qo=_view(H=4)), cg.CG_ERR_ARG), (dict(plan=_bad_plan()), cg.CG_ERR_ARG),
    (dict(rot=66), cg.CG_ERR_SHAPE), (dict(q=_view(H=4), qo=_view(H=3)), cg.CG_ERR_SHAPE),
    (dict(q=_view(H=4, T=15), qo=_view(H=4, T=15)), cg.CG_ERR_SHAPE), (dict(q=_view(H=4, B=2), qo=_view(H=4, B=2)), cg.CG_ERR_SHAPE),
    (dict(q=_view(H=4, d=72), qo=_view(H=4, d=72)), cg.CG_ERR_SHAPE), (dict(q=_view(H=4, L=2), qo=_view(H=4, L=2)), cg.CG_ERR_SHAPE),
    (dict(q=_view(H=4), qo=_view(H=4, dtype=cg.DTYPE_F32)), cg.CG_ERR_SHAPE), (dict(q=_view(H=4), qo=_view(H=4, ptr=PTR + 8)), cg.CG_ERR_ALIGN),
    (dict(q=_view(H=4), qo=_view(H=4, strides=(2048, 2048, 0, 64))), cg.CG_ERR_ARG),
    (dict(k=_view(B=2), v=_view(B=2)), cg.CG_ERR_SHAPE), (dict(v=_view(T=15)), cg.CG_ERR_SHAPE), (dict(k=_view(H=3)), cg.CG_ERR_SHAPE),
    (dict(kc=_cache(T_cap=32), vc=_cache(T_cap=32)), cg.CG_ERR_SHAPE), (dict(vc=_cache(B=5)), cg.CG_ERR_SHAPE),
    (dict(codec=cg.Codec(cg.ZFP, 4)), cg.CG_ERR_UNSUPPORTED), (dict(codec=cg.Codec(cg.BLOCK_UNIFORM, 4, 32, block_t=16)), cg.CG_ERR_ARG),
    (dict(kc=_cache(B=2 ** 25, T_cap=64), vc=_cache(B=2 ** 25, T_cap=64)), cg.CG_ERR_CAPACITY),
    (dict(k=_view(T=0, ptr=None), v=_view(T=0, ptr=None), slots=None, pos=None), cg.CG_OK),
])
def test_append_rope_refuses(kw, status):
    assert _append(**kw) == status


def _attend(q=None, out=None, cu=PTR, B=2, max_q=8, mask=PTR, words=1, pos=PTR, kc=None, vc=None, pages=PTR, max_pages=4, P=64,
            shp=None, codec=BU, lens=PTR, scale=0.1, window=0, sinks=0, ws=PTR, l0=0, l1=1, gdev=0x50000, err=None):
    cs = codec.struct()
    q, out, kc, vc = q or _view(H=4), out or _view(H=4), kc or _cache(), vc or _cache()
    pt = cg.PageTable(pages, max_pages, P)
    return cg.lib().kv_attend_tree_paged(l0, l1, C.byref(q), cu, B, max_q, mask, words, pos, C.byref(kc), C.byref(vc), C.byref(pt),
                                         gdev, shp or cg.shape(1, 2, 64, 16), C.byref(cs), lens, scale, window, sinks,
                                         C.byref(out), ws, err, None)


@pytest.mark.parametrize("kw,status", [
    (dict(cu=None), cg.CG_ERR_ARG), (dict(lens=None), cg.CG_ERR_ARG), (dict(mask=None), cg.CG_ERR_ARG), (dict(pages=None), cg.CG_ERR_ARG),
    (dict(window=9, pos=None), cg.CG_ERR_ARG), (dict(mask=PTR + 4), cg.CG_ERR_ALIGN), (dict(pos=PTR + 2), cg.CG_ERR_ALIGN),
    (dict(words=0), cg.CG_ERR_SHAPE), (dict(max_q=65), cg.CG_ERR_SHAPE), (dict(max_q=1025, words=17), cg.CG_ERR_UNSUPPORTED),
    (dict(cu=PTR + 2), cg.CG_ERR_ALIGN), (dict(err=PTR + 2), cg.CG_ERR_ALIGN), (dict(B=0), cg.CG_ERR_ARG), (dict(max_q=0), cg.CG_ERR_ARG),
    (dict(window=-1), cg.CG_ERR_ARG), (dict(sinks=-1), cg.CG_ERR_ARG), (dict(scale=math.nan), cg.CG_ERR_ARG), (dict(l1=2), cg.CG_ERR_ARG),
    (dict(q=_view(H=3), out=_view(H=3)), cg.CG_ERR_SHAPE), (dict(out=_view(H=4, T=15)), cg.CG_ERR_SHAPE),
    (dict(q=_view(H=4, ptr=PTR + 8)), cg.CG_ERR_ALIGN), (dict(P=128), cg.CG_ERR_SHAPE), (dict(max_pages=2 ** 25), cg.CG_ERR_CAPACITY),
    (dict(q=_view(), out=_view(strides=(2048, 2048, 0, 64))), cg.CG_ERR_ARG), (dict(codec=cg.Codec(cg.ZFP, 4)), cg.CG_ERR_UNSUPPORTED),
    (dict(max_pages=400, ws=None), cg.CG_ERR_ARG), (dict(max_pages=400, ws=PTR + 8), cg.CG_ERR_ALIGN),
    (dict(q=_view(H=4, T=0, ptr=None), out=_view(H=4, T=0, ptr=None), mask=None), cg.CG_OK),
])
def test_attend_tree_refuses(kw, status):
    assert _attend(**kw) == status


def test_tree_workspace_holds_every_smaller_call():
    shp = cg.shape(2, 8, 128, 128)
    n = lambda *a: cg.attend_tree_workspace_bytes(shp, *a)  # noqa: E731
    assert n(1, 16, 1, 32, 400, 64) > 0
    for k in range(5):
        big, one = (2, 4096, 64, 32, 400), [2, 4096, 64, 32, 400]
        one[k] = max(1, one[k] // 2) if k != 3 else 8
        assert n(*one[:4], one[4], 64) <= n(*big[:4], big[4], 64)
    assert n(0, 1, 1, 32, 400, 64) == 0 and n(1, 1, 1, 31, 400, 64) == 0 and n(1, 1, 1, 32, 400, 63) == 0 and n(1, 0, 1, 32, 4, 64) == 0


def test_binding_refuses_host_tensors_and_other_masks():
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    with pytest.raises(ValueError):
        cg.kv_tree_map(i32(4), i32(2), i32(1), i32(4), torch.zeros((4, 1), dtype=torch.int64))
    for bad in (torch.zeros((4, 1), dtype=torch.int32), torch.zeros((5, 1), dtype=torch.int64), torch.zeros(4, dtype=torch.int64),
                torch.zeros((2, 4), dtype=torch.int64).t()):
        with pytest.raises(ValueError):
            cg._mask("f", bad, 4)
    assert cg._mask("f", torch.zeros((4, 3), dtype=torch.int64), 4) == 3


def test_the_host_trees_are_trees():
    rng = np.random.default_rng(3)
    for kind in ("chain", "star", "forest", "roots", "near"):
        for n in (0, 1, 70):
            p = T.tree(n, kind, rng)
            m, depth = T.closure(p)
            assert len(p) == n and all(-1 <= a < i for i, a in enumerate(p))
            assert all(bin(x).count("1") == k + 1 for x, k in zip(m, depth))
