"""Sampling: what the calls refuse on the host, their scratch, and the reference's own pins."""
import ctypes
import os

import numpy as np
import pytest

from tests import sample_ref

ERR_ARG, ERR_WS = -1, -2


@pytest.fixture(scope="module")
def lib():
    from paper_2604_12989_amd.build import LIB, build_library
    if not os.path.exists(LIB):
        build_library()
    import paper_2604_12989_amd as dd
    return dd.load()


@pytest.fixture(scope="module")
def p():
    buf = ctypes.create_string_buffer(1 << 16)
    q = ctypes.cast(buf, ctypes.c_void_p)
    q.value += (-q.value) % 256
    yield q
    del buf


def _f32(*v):
    return ctypes.cast((ctypes.c_float * len(v))(*v), ctypes.c_void_p)


def _i32(*v):
    return ctypes.cast((ctypes.c_int32 * len(v))(*v), ctypes.c_void_p)


BAD_OPTIONS = [dict(tau=None), dict(tau=_f32(1.0, -0.5)), dict(tau=_f32(float("nan"), 1.0)), dict(tau=_f32(1.0, float("inf"))),
               dict(tau=_f32(2e30, 1.0)), dict(k=_i32(0, -1)), dict(top_p=_f32(1.0, 0.0)), dict(top_p=_f32(1.0, -0.0)), dict(top_p=_f32(1.5, 1.0)),
               dict(top_p=_f32(float("nan"), 1.0)), dict(top_p=_f32(-0.1, 1.0)), dict(min_p=_f32(0.0, 1.01)),
               dict(min_p=_f32(-0.1, 0.0)), dict(min_p=_f32(float("nan"), 0.0))]


def test_sample_refuses_bad_arguments(lib, p):
    odd = ctypes.c_void_p(p.value + 2)
    good = dict(x=p, batch=2, T=1, V=8, tau=_f32(1.0, 0.0), k=_i32(0, 5), top_p=_f32(0.9, 1.0), min_p=_f32(0.0, 1.0), u=p, out=p, ws=p,
                n=1 << 16)
    bad = BAD_OPTIONS + [dict(x=None), dict(u=None), dict(out=None), dict(x=odd), dict(u=odd), dict(out=odd), dict(batch=0), dict(batch=65),
                         dict(T=0), dict(T=1026), dict(V=0), dict(V=(1 << 22) + 1)]
    for change in bad:
        a = dict(good, **change)
        rc = lib.ddtree_sample(a["x"], a["batch"], a["T"], a["V"], a["tau"], a["k"], a["top_p"], a["min_p"], a["u"], a["out"], a["ws"], a["n"], None)
        assert rc == ERR_ARG, change
    for change in (dict(ws=None), dict(n=100), dict(ws=ctypes.c_void_p(p.value + 16)), dict(V=151936)):
        a = dict(good, **change)
        rc = lib.ddtree_sample(a["x"], a["batch"], a["T"], a["V"], a["tau"], a["k"], a["top_p"], a["min_p"], a["u"], a["out"], a["ws"], a["n"], None)
        assert rc == ERR_WS, change


def test_accept_filtered_refuses_bad_arguments(lib, p):
    good = dict(x=p, batch=2, T=3, V=8, tok=p, par=p, dep=p, n=p, tau=_f32(1.0, 0.0), k=None, top_p=None, min_p=None, u=p, path=p, acc=p,
                bonus=p, post=None, B=4, ws=p, nws=1 << 16)
    bad = BAD_OPTIONS + [{k: None} for k in ("x", "tok", "par", "dep", "n", "u", "path", "acc", "bonus")] + \
        [dict(T=1), dict(T=1026), dict(B=0), dict(B=33), dict(batch=0), dict(V=0)]
    for change in bad:
        a = dict(good, **change)
        rc = lib.ddtree_accept_filtered(*(a[k] for k in ("x", "batch", "T", "V", "tok", "par", "dep", "n", "tau", "k", "top_p", "min_p", "u",
                                                         "path", "acc", "bonus", "post", "B", "ws", "nws")), None)
        assert rc == ERR_ARG, change
    a = dict(good, nws=64)
    assert lib.ddtree_accept_filtered(*(a[k] for k in ("x", "batch", "T", "V", "tok", "par", "dep", "n", "tau", "k", "top_p", "min_p", "u",
                                                       "path", "acc", "bonus", "post", "B", "ws", "nws")), None) == ERR_WS


def test_the_binding_refuses_options_of_another_length():
    import paper_2604_12989_amd as dd
    from paper_2604_12989_amd import binding
    with pytest.raises(dd.DDTreeError):
        binding._options(3, [1.0, 1.0], 0, 1.0, 0.0)
    arrays, _ = binding._options(3, 0.5, [1, 2, 3], 1.0, 0.0)
    assert arrays[0].tolist() == [0.5] * 3 and arrays[1].tolist() == [1, 2, 3]


def test_reference_worked_rows():
    ln2 = np.log(2.0)
    x = np.float32([0, 2 * ln2, ln2, 0, -np.inf])             # weights 1 4 2 1 0, in quarters of the largest
    t = sample_ref.token
    assert [t(x, u, 1.0) for u in (0, 0.124, 0.126, 0.62, 0.63, 0.874, 0.876, 0.999)] == [0, 0, 1, 1, 2, 2, 3, 3]
    assert [t(x, u, 1.0, top_k=2) for u in (0, 0.66, 0.67)] == [1, 1, 2]
    assert [t(x, u, 1.0, top_k=3) for u in (0, 0.13, 0.15)] == [0, 0, 1]         # of the two equal ones the lower id is third
    assert [t(x, u, 1.0, top_p=0.4) for u in (0, 0.99)] == [1, 1]
    assert [t(x, u, 1.0, top_p=0.6) for u in (0.6, 0.7)] == [1, 2]
    assert [t(x, u, 1.0, min_p=0.3) for u in (0.6, 0.7)] == [1, 2]
    assert t(x, 0.99, 0.0) == 1 and t([-np.inf] * 3, 0.5, 1.0) == -1 and t([np.nan, 1.0], 0.0, 1.0) == 1
