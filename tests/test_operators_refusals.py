"""What the operators beside densify refuse, and their host arithmetic.  No GPU: every call here is refused, or has nothing to
do, before anything is launched; the addresses are never used."""
import ctypes as C

import pytest
import torch

from paper_1905_04035_amd import binding as ts

P = C.c_void_p(1 << 20)            # an aligned address
ODD = C.c_void_p((1 << 20) + 8)
N31 = 1 << 31


def mask(p=0.1, step=None):
    return C.byref(ts.TsDropoutMask(1, 2, step, p, 0))


def test_dropout():
    f = ts.lib().ts_dropout
    ok = [P, None, 8, 16, ts.TS_ROW_FP32, mask(), P, None]
    for at, value, want in ((0, None, ts.TS_ERR_NULL), (6, None, ts.TS_ERR_NULL), (5, None, ts.TS_ERR_NULL),
                            (2, -1, ts.TS_ERR_SHAPE), (3, 0, ts.TS_ERR_SHAPE), (3, 6, ts.TS_ERR_SHAPE), (4, 2, ts.TS_ERR_SHAPE),
                            (2, N31, ts.TS_ERR_OVERFLOW), (0, ODD, ts.TS_ERR_ALIGN), (1, ODD, ts.TS_ERR_ALIGN), (6, ODD, ts.TS_ERR_ALIGN),
                            (5, mask(step=4), ts.TS_ERR_ALIGN)):
        assert f(*[value if i == at else x for i, x in enumerate(ok)]) == want, (at, value)
    for p in (-0.1, 1.0, 1.5, float("nan"), float("inf"), float("-inf")):
        assert f(*ok[:5], mask(p), *ok[6:]) == ts.TS_ERR_SHAPE
    assert f(None, None, 0, 16, 0, mask(), None, None) == ts.TS_OK


def test_lookup_dropout():
    f = ts.lib().ts_lookup_dropout
    ok = [P, 8, P, 0, 16, 100, 1.0, P, P, 10, mask(), P, 0, None]
    for at, value, want in ((0, None, ts.TS_ERR_NULL), (2, None, ts.TS_ERR_NULL), (11, None, ts.TS_ERR_NULL), (10, None, ts.TS_ERR_NULL),
                            (8, None, ts.TS_ERR_NULL), (7, None, ts.TS_ERR_NULL),
                            (1, -1, ts.TS_ERR_SHAPE), (4, 0, ts.TS_ERR_SHAPE), (4, 18, ts.TS_ERR_SHAPE), (5, 0, ts.TS_ERR_SHAPE),
                            (9, -1, ts.TS_ERR_SHAPE), (3, 2, ts.TS_ERR_SHAPE), (12, 2, ts.TS_ERR_SHAPE), (6, float("nan"), ts.TS_ERR_SHAPE),
                            (6, float("inf"), ts.TS_ERR_SHAPE), (10, mask(1.0), ts.TS_ERR_SHAPE),
                            (1, N31, ts.TS_ERR_OVERFLOW), (4, 1 << 24, ts.TS_ERR_OVERFLOW),
                            (2, ODD, ts.TS_ERR_ALIGN), (7, ODD, ts.TS_ERR_ALIGN), (11, ODD, ts.TS_ERR_ALIGN),
                            (0, C.c_void_p(2), ts.TS_ERR_ALIGN), (8, C.c_void_p(2), ts.TS_ERR_ALIGN)):
        assert f(*[value if i == at else x for i, x in enumerate(ok)]) == want, (at, value)
    assert f(None, 0, None, 0, 16, 100, 1.0, None, None, 0, mask(), None, 0, None) == ts.TS_OK


def test_densify_dropout():
    f = ts.lib().ts_densify_dropout
    ts.lib().ts_bind_workspace(None, 0)
    ok = [P, P, 8, 0, 16, 100, 2.0, mask(), P, P, None]
    for at, value, want in ((0, None, ts.TS_ERR_NULL), (1, None, ts.TS_ERR_NULL), (7, None, ts.TS_ERR_NULL), (9, None, ts.TS_ERR_NULL),
                            (2, -1, ts.TS_ERR_SHAPE), (3, 2, ts.TS_ERR_SHAPE), (4, 6, ts.TS_ERR_SHAPE), (5, 0, ts.TS_ERR_SHAPE),
                            (6, float("nan"), ts.TS_ERR_SHAPE), (6, float("-inf"), ts.TS_ERR_SHAPE), (6, 3.4e38, ts.TS_ERR_SHAPE),
                            (7, mask(-0.5), ts.TS_ERR_SHAPE), (2, N31, ts.TS_ERR_OVERFLOW), (1, ODD, ts.TS_ERR_ALIGN),
                            (8, ODD, ts.TS_ERR_ALIGN), (9, ODD, ts.TS_ERR_ALIGN)):
        assert f(*[value if i == at else x for i, x in enumerate(ok)]) == want, (at, value)
    assert f(*ok) == ts.TS_ERR_WORKSPACE                              # none is bound


def test_layout():
    assert [ts.ts_fp8_layout(k) for k in (0, 1, 127, 128, 129, 512, 513, 32768)] == [
        (0, 0), (128, 4), (128, 4), (128, 4), (256, 4), (512, 4), (640, 8), (32768, 256)]
    f, a, b = ts.lib().ts_fp8_layout, C.c_int64(), C.c_int64()
    assert f(1, None, C.byref(b)) == ts.TS_ERR_NULL and f(1, C.byref(a), None) == ts.TS_ERR_NULL
    assert f(-1, C.byref(a), C.byref(b)) == ts.TS_ERR_SHAPE and f(N31, C.byref(a), C.byref(b)) == ts.TS_ERR_OVERFLOW


def test_quantize():
    f = ts.lib().ts_quantize_fp8
    ok = [P, 0, 8, 16, 0, P, P, P, P, None]
    for at, value, want in ((0, None, ts.TS_ERR_NULL), (5, None, ts.TS_ERR_NULL), (6, None, ts.TS_ERR_NULL), (7, None, ts.TS_ERR_NULL),
                            (8, None, ts.TS_ERR_NULL), (1, 2, ts.TS_ERR_SHAPE), (2, -1, ts.TS_ERR_SHAPE), (3, -1, ts.TS_ERR_SHAPE),
                            (4, 2, ts.TS_ERR_SHAPE), (2, N31, ts.TS_ERR_OVERFLOW), (3, N31, ts.TS_ERR_OVERFLOW),
                            (0, ODD, ts.TS_ERR_ALIGN), (5, ODD, ts.TS_ERR_ALIGN), (7, ODD, ts.TS_ERR_ALIGN),
                            (6, C.c_void_p(2), ts.TS_ERR_ALIGN), (8, C.c_void_p(2), ts.TS_ERR_ALIGN)):
        assert f(*[value if i == at else x for i, x in enumerate(ok)]) == want, (at, value)
    assert f(P, 0, 8, 16, 0, None, None, None, None, None) == ts.TS_ERR_NULL
    assert f(None, 0, 0, 16, 0, P, P, None, None, None) == ts.TS_OK and f(None, 0, 8, 0, 0, None, None, P, P, None) == ts.TS_OK
    assert f(None, 0, 0, 0, 0, P, P, None, None, None) == ts.TS_OK and f(None, 0, 8, 0, 2, P, P, None, None, None) == ts.TS_ERR_SHAPE
    assert f(None, 0, 8, 0, 0, None, None, None, None, None) == ts.TS_OK          # (empty tensors have no addresses)


def test_matmul():
    f = ts.lib().ts_matmul_fp8
    ok = [P, P, 0, P, P, 1, 8, 16, 32, P, P, 0, None]
    for at, value, want in ((0, None, ts.TS_ERR_NULL), (1, None, ts.TS_ERR_NULL), (3, None, ts.TS_ERR_NULL), (4, None, ts.TS_ERR_NULL),
                            (10, None, ts.TS_ERR_NULL), (2, 2, ts.TS_ERR_SHAPE), (5, -1, ts.TS_ERR_SHAPE), (6, -1, ts.TS_ERR_SHAPE),
                            (7, -1, ts.TS_ERR_SHAPE), (8, -1, ts.TS_ERR_SHAPE), (11, 2, ts.TS_ERR_SHAPE), (11, 1, ts.TS_ERR_SHAPE),
                            (6, N31, ts.TS_ERR_OVERFLOW), (7, N31, ts.TS_ERR_OVERFLOW), (8, (1 << 24) - 127, ts.TS_ERR_OVERFLOW),
                            (0, ODD, ts.TS_ERR_ALIGN), (3, ODD, ts.TS_ERR_ALIGN), (9, ODD, ts.TS_ERR_ALIGN), (10, ODD, ts.TS_ERR_ALIGN),
                            (1, C.c_void_p(2), ts.TS_ERR_ALIGN), (4, C.c_void_p(2), ts.TS_ERR_ALIGN)):
        assert f(*[value if i == at else x for i, x in enumerate(ok)]) == want, (at, value)
    assert f(None, None, 0, None, None, 0, 0, 16, 32, None, None, 0, None) == ts.TS_OK
    assert f(None, None, 0, None, None, 0, 16, 0, 32, None, None, 0, None) == ts.TS_OK


def test_matmul_workspace_bytes():
    f, b = ts.lib().ts_matmul_workspace_bytes, C.c_int64(-1)
    assert f(1, 1, 1, None) == ts.TS_ERR_NULL
    for sizes, want in (((-1, 1, 1), ts.TS_ERR_SHAPE), ((1, -1, 1), ts.TS_ERR_SHAPE), ((1, 1, -1), ts.TS_ERR_SHAPE),
                        ((N31, 1, 1), ts.TS_ERR_OVERFLOW), ((1, N31, 1), ts.TS_ERR_OVERFLOW), ((1, 1, (1 << 24) - 127), ts.TS_ERR_OVERFLOW)):
        assert f(*sizes, C.byref(b)) == want
    for sizes in ((0, 0, 0), (1, 32768, 1024), (8192, 32768, 1024), (64, 1024, 32768), (1, 1, (1 << 24) - 128), (16, 16, 100)):
        assert 0 <= ts.ts_matmul_workspace_bytes(*sizes) < 1 << 31


def test_tensors_that_are_not_on_the_gpu_are_refused():
    t, ids, m = torch.zeros(8, 16), torch.zeros(8, dtype=torch.int32), ts.DropoutMask(0.1, 1)
    q, s = ts.fp8_empty(8, 16, device="cpu")
    for call in (lambda: ts.ts_dropout(t, m, t), lambda: ts.ts_lookup_dropout(ids, t, 1.0, m, t),
                 lambda: ts.ts_densify_dropout(ids, t, 16, 8, 1.0, m, t, t), lambda: ts.ts_quantize_fp8(t, 0, q, s),
                 lambda: ts.ts_matmul_fp8(q, s, q, s, 16, torch.zeros(8, 8))):
        with pytest.raises(AssertionError):
            call()


def test_what_is_no_tensor():
    t, m = torch.zeros(8, 16), ts.DropoutMask(0.1, 1)
    for call in (lambda: ts.ts_dropout([1.0], m, t), lambda: ts.ts_lookup_dropout(None, t, 1.0, m, t),
                 lambda: ts.ts_densify_dropout("ids", t, 16, 8, 1.0, m, t, t), lambda: ts.ts_quantize_fp8(3, 0, t, t),
                 lambda: ts.ts_matmul_fp8(t, t, t, t, 16, None)):
        with pytest.raises(TypeError):
            call()
