"""What the calls on a 4-bit cache refuse, on the host and before anything is launched; and the format's reference."""
import ctypes

import numpy as np
import pytest

from tests import q4_ref

ERR_ARG = -1


@pytest.fixture(scope="module")
def lib():
    import os
    from paper_2604_12989_amd.build import LIB, build_library
    if not os.path.exists(LIB):
        build_library()
    import paper_2604_12989_amd as dd
    return dd.load()


def _p(buf):
    p = ctypes.cast(buf, ctypes.c_void_p)
    p.value += (-p.value) % 256
    return p


def _i32(*v):
    return ctypes.cast((ctypes.c_int32 * len(v))(*v), ctypes.c_void_p)


@pytest.fixture(scope="module")
def p():
    buf = ctypes.create_string_buffer(4096)
    yield _p(buf)
    del buf


def test_store_and_load_refuse_bad_arguments(lib, p):
    off4 = ctypes.c_void_p(p.value + 4)
    off1 = ctypes.c_void_p(p.value + 1)
    good = dict(k=p, v=p, off=_i32(0, 5), row=_i32(3), batch=1, Hkv=2, D=64, dtype=0, kc=p, ks=p, vc=p, vs=p, rows=8)
    bad = [dict(k=None), dict(v=None), dict(k=off4), dict(v=off4), dict(off=None), dict(row=None), dict(batch=0), dict(batch=65),
           dict(Hkv=0), dict(Hkv=40000), dict(D=48), dict(D=0), dict(D=288), dict(dtype=2), dict(kc=None), dict(ks=None),
           dict(vc=None), dict(vs=None), dict(kc=off4), dict(vc=off4), dict(ks=off1), dict(vs=off1), dict(rows=0),
           dict(rows=7), dict(row=_i32(-1)), dict(row=_i32(4)), dict(off=_i32(-1, 2)), dict(off=_i32(4, 2)),
           dict(row=_i32(0x7FFFFFFF)), dict(off=_i32(0, 0x7FFFFFFF), rows=0x7FFFFFFF, row=_i32(0))]
    for change in bad:
        a = dict(good, **change)
        store = lib.ddtree_q4_store(a["k"], a["v"], a["off"], a["row"], a["batch"], a["Hkv"], a["D"], a["dtype"], a["kc"], a["ks"],
                                    a["vc"], a["vs"], a["rows"], None)
        load = lib.ddtree_q4_load(a["kc"], a["ks"], a["vc"], a["vs"], a["rows"], a["row"], a["off"], a["batch"], a["Hkv"], a["D"],
                                  a["dtype"], a["k"], a["v"], None)
        assert (store, load) == (ERR_ARG, ERR_ARG), change


def test_nothing_to_store_or_load_is_no_error(lib, p):
    assert lib.ddtree_q4_store(None, None, _i32(5, 5), _i32(8), 1, 2, 64, 0, p, p, p, p, 8, None) == 0
    assert lib.ddtree_q4_load(p, p, p, p, 8, _i32(8), _i32(0, 0), 1, 2, 64, 1, None, None, None) == 0


def test_append_refuses_bad_arguments(lib, p):
    off4 = ctypes.c_void_p(p.value + 4)
    good = dict(k=p, v=p, path=p, n=p, row=_i32(3), batch=1, T=5, B=4, Hkv=2, D=64, dtype=0, kc=p, ks=p, vc=p, vs=p, rows=8)
    bad = [dict(k=None), dict(v=None), dict(k=off4), dict(path=None), dict(n=None), dict(row=None), dict(batch=0), dict(batch=65),
           dict(T=0), dict(T=1026), dict(B=0), dict(B=33), dict(Hkv=0), dict(D=100), dict(dtype=-1), dict(kc=None), dict(vs=None),
           dict(rows=7), dict(row=_i32(-1)), dict(row=_i32(4)), dict(row=_i32(0x7FFFFFFF))]
    for change in bad:
        a = dict(good, **change)
        rc = lib.ddtree_q4_append(a["k"], a["v"], a["path"], a["n"], a["row"], a["batch"], a["T"], a["B"], a["Hkv"], a["D"], a["dtype"],
                                  a["kc"], a["ks"], a["vc"], a["vs"], a["rows"], None)
        assert rc == ERR_ARG, change


def test_rows_of_two_sequences_are_refused(lib, p):
    """Codes and scales of one row could come from either."""
    for off, row, rc in [((0, 5, 9), (3, 7), ERR_ARG), ((0, 5, 9), (7, 10), ERR_ARG), ((0, 5, 9), (3, 3), ERR_ARG),
                         ((0, 0, 0), (3, 3), 0), ((2, 2, 2), (12, 3), 0)]:
        assert lib.ddtree_q4_store(p, p, _i32(*off), _i32(*row), 2, 2, 64, 0, p, p, p, p, 12, None) == rc, (off, row)
    for row in [(3, 3, 20), (3, 20, 7), (7, 20, 3), (20, 3, 16)]:
        assert lib.ddtree_q4_append(p, p, p, p, _i32(*row), 3, 5, 4, 2, 64, 0, p, p, p, p, 25, None) == ERR_ARG, row


def test_the_binding_refuses_tensors_that_are_no_cache():
    import torch
    import paper_2604_12989_amd as dd
    u8 = torch.zeros((2, 8, 32), dtype=torch.uint8)
    with pytest.raises(dd.DDTreeError):
        dd.CacheQ4(u8, u8[:, :, :2], u8, u8[:, :, :2])      # on the host


def test_reference_of_the_format():
    """Worked blocks: the largest magnitude decides the power of two, its neighbours round to the even code."""
    x = np.zeros((1, 64))
    x[0, :8] = [7.0, 6.9, -5.0, 2.5, 0.25, 0.26, -0.75, 3.5]          # 7 is a tie between 6 and 8: the unit is 2
    x[0, 32:40] = [6.99, 5.0, -5.01, 2.5, 0.25, 0.26, -0.75, 3.5]     # the unit is 1
    codes, scales = q4_ref.encode(x)
    assert scales.tolist() == [[128, 127]]
    back = q4_ref.decode(codes, scales)[0]
    assert back[:8].tolist() == [8.0, 6.0, -4.0, 2.0, 0.0, 0.0, -1.0, 4.0]
    assert back[32:40].tolist() == [6.0, 4.0, -6.0, 2.0, 0.0, 0.5, -1.0, 4.0]
    for c in range(256):                                              # each code of each half, once around
        code = np.full((1, 16), c, np.uint8)
        v = q4_ref.decode(code, np.array([[127]], np.uint8))
        if np.abs(v).max() >= 4.0:
            again, s = q4_ref.encode(v)
            assert np.array_equal(again, code) and s[0, 0] == 127


def test_attention_refuses_bad_arguments(lib, p):
    off4, off1 = ctypes.c_void_p(p.value + 4), ctypes.c_void_p(p.value + 1)
    good = dict(q=p, kc=p, ks=p, vc=p, vs=p, rows=8, kt=p, vt=p, mask=p, start=_i32(3), len=_i32(5), batch=1, T=5, Hq=4, Hkv=2, D=64,
                scale=0.125, dtype=1, out=p)
    bad = [dict(q=None), dict(kt=None), dict(vt=None), dict(mask=None), dict(out=None), dict(start=None), dict(len=None), dict(kc=None),
           dict(ks=None), dict(vc=None), dict(vs=None), dict(kc=off4), dict(vs=off1), dict(q=off4), dict(out=off4), dict(mask=off4),
           dict(batch=0), dict(batch=65), dict(T=0), dict(T=1026), dict(Hq=3), dict(Hkv=0), dict(D=40), dict(D=288), dict(D=16),
           dict(scale=0.0), dict(scale=float("nan")), dict(dtype=2), dict(rows=7), dict(rows=0), dict(start=_i32(-1)), dict(len=_i32(-1)),
           dict(start=_i32(4)), dict(start=_i32(0x7FFFFFFF))]
    for change in bad:
        a = dict(good, **change)
        rc = lib.ddtree_verify_attn_q4(a["q"], a["kc"], a["ks"], a["vc"], a["vs"], a["rows"], a["kt"], a["vt"], a["mask"], a["start"],
                                       a["len"], a["batch"], a["T"], a["Hq"], a["Hkv"], a["D"], a["scale"], a["dtype"], a["out"], None, 0, None)
        assert rc == ERR_ARG, change
    # a long key range that few workgroups share wants its scratch, as over a bf16 cache
    assert lib.ddtree_verify_attn_q4(p, p, p, p, p, 8192, p, p, p, _i32(0), _i32(8192), 1, 257, 32, 8, 128, 0.088, 0, p, None, 0, None) == -2
