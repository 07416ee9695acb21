"""Refusals of the calls on a cache that grows and shrinks: on the host, before anything is launched.  No GPU needed."""
import ctypes

import pytest

from paper_2503_18893_amd import binding as xb

NULL, AL = ctypes.c_void_p(0), ctypes.c_void_p(4096)  # never dereferenced
BIG = 1 << 40


def shape(**kw):
    f = dict(G=1, H_kv=8, H_q=32, d_h=128, r_k=1, r_v=1, L=1000, k=100, batch=2, dtype="bf16")
    f.update(kw)
    return xb.Shape(**f)


def tree(s, N=4, ws=AL, size=BIG, **null):
    a = {x: NULL if x in null else AL for x in ("K", "V", "lengths", "q", "Kd", "Vd", "tree", "out")}
    return xb.load().xkv_tree_decode(ctypes.byref(s.c()), a["K"], a["V"], a["lengths"], a["q"], a["Kd"], a["Vd"], a["tree"], N, a["out"], ws,
                                     size, NULL)


def block(s, N=1, c=16, ws=AL, size=BIG, **null):
    a = {x: NULL if x in null else AL for x in ("K", "V", "visible", "q", "marks", "out", "blocks")}
    return xb.load().xkv_block_decode(ctypes.byref(s.c()), a["K"], a["V"], a["visible"], a["q"], N, a["marks"], c, a["out"], a["blocks"], ws,
                                      size, NULL)


def weights(s, ws=AL, size=BIG, **null):
    a = {x: NULL if x in null else AL for x in ("K", "V", "lengths", "q", "out", "weights")}
    return xb.load().xkv_dense_decode_weights(ctypes.byref(s.c()), a["K"], a["V"], a["lengths"], a["q"], a["out"], a["weights"], ws, size, NULL)


def evict(s, sink=4, recent=10, L_out=100, ws=AL, size=BIG, **other):
    a = dict(K=1 << 20, V=2 << 20, w=3 << 20, K_out=4 << 20, V_out=5 << 20, w_out=6 << 20)
    a.update(other)
    p = {x: ctypes.c_void_p(v) for x, v in a.items()}
    return xb.load().xkv_evict(ctypes.byref(s.c()), p["K"], p["V"], p["w"], AL, sink, recent, L_out, p["K_out"], p["V_out"], p["w_out"], NULL,
                               NULL, ws, size, NULL)


def update(s, N=1, c=16, K=AL, marks=AL):
    return xb.load().xkv_landmarks_update(ctypes.byref(s.c()), K, NULL, N, c, marks, NULL)


def test_missing_operands_are_refused():
    s = shape()
    for x in ("K", "V", "q", "Kd", "Vd", "out"):
        assert tree(s, **{x: 1}) == xb.XKV_ERR_INVALID_ARG, x
    for x in ("K", "V", "q", "marks", "out"):
        assert block(s, **{x: 1}) == xb.XKV_ERR_INVALID_ARG, x
    for x in ("K", "V", "q", "out", "weights"):
        assert weights(s, **{x: 1}) == xb.XKV_ERR_INVALID_ARG, x
    for x in ("K", "V", "w", "K_out", "V_out", "w_out"):
        assert evict(s, **{x: 0}) == xb.XKV_ERR_INVALID_ARG, x
    assert update(s, K=NULL) == update(s, marks=NULL) == xb.XKV_ERR_INVALID_ARG


@pytest.mark.parametrize("call", [tree, block, weights, evict])
def test_workspaces_are_checked(call):
    s = shape()
    assert call(s, ws=NULL) == xb.XKV_ERR_INVALID_ARG
    assert call(s, ws=ctypes.c_void_p(4096 + 128)) == xb.XKV_ERR_INVALID_ARG
    assert call(s, size=64) == xb.XKV_ERR_WORKSPACE


@pytest.mark.parametrize("call", [tree, block, weights, evict, update])
def test_bad_shapes_are_refused(call):
    for kw in (dict(H_q=30), dict(batch=-1), dict(L=0, k=1), dict(k=0), dict(scale=-1.0)):
        assert call(shape(**kw)) == xb.XKV_ERR_INVALID_ARG, kw
    for kw in (dict(d_h=257), dict(H_q=8 * 17)):
        assert call(shape(**kw)) == xb.XKV_ERR_UNSUPPORTED, kw
    assert call(shape(batch=0)) == xb.XKV_OK  # nothing to do


def test_counts_are_checked():
    s = shape()
    assert tree(s, N=0) == block(s, N=0) == update(s, N=0) == xb.XKV_ERR_INVALID_ARG
    assert block(s, c=0) == block(s, c=-1) == update(s, c=0) == xb.XKV_ERR_INVALID_ARG
    assert tree(s, N=1025) == xb.XKV_ERR_UNSUPPORTED
    assert block(s, N=5000) == xb.XKV_ERR_UNSUPPORTED          # 2 * 5000 * 8 rows of the selection
    assert tree(shape(batch=100), N=100) == xb.XKV_ERR_UNSUPPORTED
    long = shape(L=2 ** 30 + 1)
    assert tree(long) == block(long) == weights(long) == xb.XKV_ERR_UNSUPPORTED


def test_caches_that_are_too_long_are_refused():
    for call in (tree, block, weights, evict, update):
        assert call(shape(L=2 ** 30 + 1)) == xb.XKV_ERR_UNSUPPORTED, call.__name__
        assert call(shape(L=2 ** 31 - 1)) == xb.XKV_ERR_UNSUPPORTED, call.__name__


def test_evictions_are_checked():
    s = shape()
    assert evict(s, sink=-1) == evict(s, recent=-1) == xb.XKV_ERR_INVALID_ARG
    assert evict(s, sink=60, recent=41) == xb.XKV_ERR_INVALID_ARG     # more than k
    assert evict(s, sink=2 ** 31 - 1, recent=2 ** 31 - 1) == xb.XKV_ERR_INVALID_ARG
    assert evict(s, L_out=99) == xb.XKV_ERR_INVALID_ARG
    assert evict(s, K_out=1 << 20, L_out=1000) == xb.XKV_ERR_INVALID_ARG                 # keys in place, the rest not
    assert evict(s, K_out=1 << 20, V_out=2 << 20, w_out=3 << 20, L_out=999) == xb.XKV_ERR_INVALID_ARG


def test_workspace_sizes():
    s = shape()
    n = ctypes.c_size_t(0)
    f = xb.load().xkv_cache_workspace_bytes
    assert xb.xkv_cache_workspace_bytes(s, 64, 16) >= xb.xkv_cache_workspace_bytes(s, 64) >= 2 * 32 * 1000 * 4
    assert f(ctypes.byref(s.c()), 0, 0, ctypes.byref(n)) == f(ctypes.byref(s.c()), 1, -1, ctypes.byref(n)) == xb.XKV_ERR_INVALID_ARG
    assert f(ctypes.byref(s.c()), 1, 0, None) == f(None, 1, 0, ctypes.byref(n)) == xb.XKV_ERR_INVALID_ARG
    assert f(ctypes.byref(s.c()), 1025, 0, ctypes.byref(n)) == xb.XKV_ERR_UNSUPPORTED    # no tree of that many, and no blocks asked for
    assert f(ctypes.byref(s.c()), 1025, 16, ctypes.byref(n)) == xb.XKV_OK                # a prompt's queries
