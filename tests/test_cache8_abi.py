"""Refusals of rotary positions and of the calls on a cache held in 8 bits: on the host, before anything is launched.  No GPU needed."""
import ctypes

import pytest

from paper_2503_18893_amd import binding as xb

NULL, AL = ctypes.c_void_p(0), ctypes.c_void_p(4096)  # never dereferenced
BIG = 1 << 44
BAD, CANNOT = xb.XKV_ERR_INVALID_ARG, xb.XKV_ERR_UNSUPPORTED


def shape(**kw):
    f = dict(G=1, H_kv=8, H_q=32, d_h=128, r_k=1, r_v=1, L=1000, k=100, batch=2, dtype="bf16")
    f.update(kw)
    return xb.Shape(**f)


def at(*strides):
    return ctypes.byref(xb.xkv_rows(*strides))


def rotate(s, d_rot=128, layout=0, direction=0, amplitude=1.0, N=4, q_at=None, q_out_at=None, K_at=None, K_out_at=None, **null):
    p = dict(f=1 << 20, q=2 << 20, q_out=3 << 20, K=4 << 20, K_out=5 << 20)
    p.update(null)
    v = {x: ctypes.c_void_p(y) for x, y in p.items()}
    return xb.load().xkv_rotate(ctypes.byref(s.c()), d_rot, layout, direction, amplitude, v["f"], NULL, N, v["q"], q_at, v["q_out"], q_out_at,
                                v["K"], K_at, v["K_out"], K_out_at, NULL)


def append(s, N=4, code=0, c=16, K_at=None, V_at=None, **null):
    v = {x: NULL if x in null else AL for x in ("K", "V", "K8", "V8", "ks", "vs")}
    return xb.load().xkv_cache8_append(ctypes.byref(s.c()), v["K"], K_at, v["V"], V_at, NULL, NULL, N, code, c, v["K8"], v["V8"], v["ks"],
                                       v["vs"], NULL)


def decode(s, N=1, code=0, c=16, ws=AL, size=BIG, **null):
    v = {x: NULL if x in null else AL for x in ("K8", "V8", "ks", "vs", "q", "out")}
    return xb.load().xkv_cache8_decode(ctypes.byref(s.c()), v["K8"], v["V8"], v["ks"], v["vs"], code, c, NULL, v["q"], N, v["out"], ws, size,
                                       NULL)


def frequencies(d_rot=128, theta=1e4, scaling=0, factor=2.0, low=1.0, high=4.0, context=8192.0, to=NULL):
    return xb.load().xkv_rope_frequencies(d_rot, theta, scaling, factor, low, high, context, to, NULL)


@pytest.mark.parametrize("call", [rotate, append, decode])
def test_bad_shapes_are_refused(call):
    for kw in (dict(H_q=30), dict(batch=-1), dict(L=0, k=1), dict(k=0), dict(scale=-1.0)):
        assert call(shape(**kw)) == BAD, kw
    for kw in (dict(d_h=257), dict(H_q=8 * 17)):
        assert call(shape(**kw)) == CANNOT, kw
    assert call(shape(), N=0) == call(shape(), N=-3) == BAD
    assert call(shape(batch=0)) == xb.XKV_OK  # nothing to do


def test_missing_operands_are_refused():
    s = shape()
    for x in ("K", "V", "K8", "V8", "ks", "vs"):
        assert append(s, **{x: 1}) == BAD, x
    for x in ("K8", "V8", "ks", "vs", "q", "out"):
        assert decode(s, **{x: 1}) == BAD, x
    for x in ("f", "q", "q_out", "K", "K_out"):
        assert rotate(s, **{x: 0}) == BAD, x
    assert rotate(s, q=0, q_out=0, K=0, K_out=0) == BAD
    assert rotate(shape(batch=0), q=0, q_out=0) == rotate(shape(batch=0), K=0, K_out=0) == xb.XKV_OK
    assert frequencies() == BAD


def test_workspaces_are_checked():
    s = shape()
    assert decode(s, ws=NULL) == decode(s, ws=ctypes.c_void_p(4096 + 128)) == BAD
    need = xb.xkv_cache8_workspace_bytes(s, 1)
    assert decode(s, size=need - 1) == xb.XKV_ERR_WORKSPACE
    assert xb.load().xkv_cache8_workspace_bytes(ctypes.byref(s.c()), 1, None) == BAD
    n = ctypes.c_size_t(0)
    assert xb.load().xkv_cache8_workspace_bytes(ctypes.byref(s.c()), 0, ctypes.byref(n)) == BAD
    assert xb.load().xkv_cache8_workspace_bytes(ctypes.byref(s.c()), 1 << 22, ctypes.byref(n)) == CANNOT


def test_codes_and_blocks_are_checked():
    s = shape()
    for call in (append, decode):
        assert call(s, code=2) == call(s, code=-1) == call(s, c=0) == call(s, c=-16) == BAD
        assert call(s, c=3) == call(s, c=24) == call(shape(L=(1 << 30) + 1)) == CANNOT
        assert call(shape(batch=0), c=1) == call(shape(batch=0), c=1 << 30) == xb.XKV_OK
    assert append(shape(L=1 << 30, batch=64), N=1 << 30, c=1) == CANNOT
    assert decode(s, N=1 << 21) == CANNOT  # 2^27 rows of queries


def test_rotations_are_checked():
    s = shape()
    assert rotate(s, d_rot=0) == rotate(s, d_rot=-2) == rotate(s, d_rot=7) == rotate(s, d_rot=130) == BAD
    assert rotate(s, layout=2) == rotate(s, layout=-1) == rotate(s, direction=3) == rotate(s, direction=-1) == BAD
    for m in (-1.0, float("inf"), float("nan"), 1e-40):
        assert rotate(s, amplitude=m) == BAD, m
    assert rotate(s, N=1 << 30) == CANNOT
    assert frequencies(to=AL, d_rot=3) == frequencies(to=AL, d_rot=0) == frequencies(to=AL, d_rot=258) == BAD
    assert frequencies(to=AL, theta=0.0) == frequencies(to=AL, theta=float("inf")) == frequencies(to=AL, theta=-1.0) == BAD
    assert frequencies(to=AL, scaling=4) == frequencies(to=AL, scaling=-1) == BAD
    for kind in (1, 2, 3):
        assert frequencies(to=AL, scaling=kind, factor=0.0) == frequencies(to=AL, scaling=kind, factor=float("nan")) == BAD
    assert frequencies(to=AL, scaling=2, d_rot=2) == BAD
    for kw in (dict(low=4.0), dict(low=-1.0), dict(context=0.0), dict(high=float("inf")), dict(low=float("nan"))):
        assert frequencies(to=AL, scaling=3, **kw) == BAD, kw


def test_strides_are_checked():
    s = shape()
    for name in ("q_at", "q_out_at", "K_at", "K_out_at"):
        assert rotate(s, **{name: at(-1, 4096, 128)}) == BAD
    assert append(s, K_at=at(0, -1, 0)) == append(s, V_at=at(0, 0, -128)) == BAD
    # outputs whose rows overlap; inputs may
    for bad in ((0, 0, 0), (4 * 32 * 128, 32 * 128, 127), (4 * 32 * 128, 32 * 128 - 1, 128), (4 * 32 * 128 - 1, 32 * 128, 128), (128, 128, 128)):
        assert rotate(s, q_out_at=at(*bad)) == BAD, bad
        assert rotate(shape(batch=0), q_at=at(*bad)) == xb.XKV_OK, bad
    # heads before tokens; one token, so that its stride is nothing
    s0 = shape(batch=0)
    assert rotate(s0, K_out_at=at(8 * 4 * 128, 128, 4 * 128)) == xb.XKV_OK
    assert rotate(s0, N=1, K_out_at=at(8 * 128, 0, 128)) == xb.XKV_OK
    # in place: as it lies
    assert rotate(s, q_out=2 << 20, q_at=at(4 * 48 * 128, 48 * 128, 128)) == BAD
    assert rotate(s0, q_out=2 << 20, q_at=at(4 * 48 * 128, 48 * 128, 128), q_out_at=at(4 * 48 * 128, 48 * 128, 128)) == xb.XKV_OK


def test_the_binding_wants_rows():
    import torch
    s, f = shape(batch=0), torch.zeros(64, dtype=torch.float64)
    x = torch.zeros((1, 2, 8, 128), dtype=torch.bfloat16)
    xb.xkv_rotate(s, 128, "half", "forward", 1.0, f, None, 2, None, None, x, x, stream=0)
    for bad in (x[0], x[:, :, :, ::2], x.transpose(2, 3)):
        with pytest.raises(ValueError):
            xb.xkv_rotate(s, 128, "half", "forward", 1.0, f, None, 2, None, None, bad, x, stream=0)
        with pytest.raises(ValueError):
            xb.xkv_cache8_append(s, x, bad, None, None, 2, "int8", 16, x, x, f, f, stream=0)
    for name in ("halves", 0):
        with pytest.raises(KeyError):
            xb.xkv_rotate(s, 128, name, "forward", 1.0, f, None, 2, None, None, x, x, stream=0)
    with pytest.raises(xb.XkvError):
        xb.xkv_rotate(shape(), 128, "half", "forward", 1.0, f, None, 0, None, None, x, x, stream=0)


def test_a_shape_that_was_used_can_be_copied_and_pickled():
    """It goes to worker processes, or into a checkpoint's configuration, before and after calls alike."""
    import copy
    import dataclasses
    import pickle
    s = shape(scale=0.25)
    xb.xkv_cache8_workspace_bytes(s, 3)
    for other in (pickle.loads(pickle.dumps(s)), copy.deepcopy(s), copy.copy(s), dataclasses.replace(s)):
        assert other == s and hash(other) == hash(s) and other is not s
        assert vars(other) == dataclasses.asdict(s)
        assert xb.xkv_cache8_workspace_bytes(other, 3) == xb.xkv_cache8_workspace_bytes(s, 3)
