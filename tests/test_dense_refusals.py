"""Arguments that the operators' C entry points refuse before they touch a GPU."""
import ctypes as C

import pytest


def lib():
    from paper_2305_01515_amd import dense
    return dense._lib()


def test_scan():
    l, h = lib(), C.c_void_p()
    for dim, dtype, bags, rows, code in ((0, 0, 1, 1, -1), (65537, 0, 1, 1, -1), (8, 3, 1, 1, -1), (8, -1, 1, 1, -1), (8, 0, -1, 1, -1), (8, 0, 1, -1, -1),
                                         (65536, 0, 1, 1 << 40, -5), (65536, 0, 1 << 40, 1, -5)):
        assert l.tbe_scan_create(C.byref(h), dim, dtype, 1, bags, rows) == code and not h
    assert l.tbe_scan_create(None, 8, 0, 1, 1, 1) == -1
    assert l.tbe_scan_forward(None, None, 8, None, 8, None, 1, 1, None, 0, None, 8, None, None, None) == -1
    assert l.tbe_scan_backward(None, None, 8, None, 8, None, 1, 1, None, 0, None, None, 8, None, None, 8, None, 8, None, None) == -1
    assert l.tbe_scan_step(None, None, 8, 1, None, None, 8, None, 8, 1, None, 8, None) == -1
    assert l.tbe_scan_saved_floats(None, 1) == -1 and l.tbe_scan_check(None, None) == -1 and l.tbe_scan_destroy(None) == 0
    assert b"null handle" in l.tbe_last_error(None)


def test_bias():
    from paper_2305_01515_amd.dense import BiasShape, BiasStrides
    l, h = lib(), C.c_void_p()
    for heads, thr in ((0, [1]), (4097, [1]), (1, [0]), (1, [2, 2]), (1, [3, 1]), (1, [-1]), (1, list(range(1, 129)))):
        assert l.tbe_bias_create(C.byref(h), heads, (C.c_int64 * len(thr))(*thr), len(thr), 0) == -1 and not h
    assert l.tbe_bias_create(C.byref(h), 1, None, 1, 0) == -1
    assert l.tbe_bias_create(None, 1, None, 0, 0) == -1
    s, t = BiasShape(), BiasStrides()
    assert l.tbe_bias_forward(None, C.byref(s), None, 0, None, None, 1.0, 0.0, None, C.byref(t), None) == -1
    assert l.tbe_bias_backward(None, C.byref(s), None, C.byref(t), None, 1.0, None, None, None) == -1
    assert l.tbe_bias_destroy(None) == 0


def test_adamw():
    from paper_2305_01515_amd.dense import AdamWTensor
    l, h = lib(), C.c_void_p()
    fine = dict(param=16, m=16, v=16, numel=4)
    for change, code in ((dict(numel=-1), -1), (dict(numel=(1 << 40) + 1), -5), (dict(param=None), -1), (dict(m=None), -1), (dict(v=None), -1),
                         (dict(param_dtype=7), -1), (dict(grad_dtype=-2), -1), (dict(weight_decay=float("nan")), -1)):
        t = (AdamWTensor * 1)(AdamWTensor(**dict(fine, **change)))
        assert l.tbe_adamw_create(C.byref(h), t, 1, 32) == code and not h
    t = (AdamWTensor * 1)(AdamWTensor(**fine))
    for n, bits in ((0, 32), (1, 16), (1, 8)):  # states in 8 bits without scales
        assert l.tbe_adamw_create(C.byref(h), t, n, bits) == -1 and not h
    assert l.tbe_adamw_create(C.byref(h), None, 1, 32) == -1
    assert l.tbe_adamw_step(None, None, 1, 0.0, 0.9, 0.9, 0.0, 0, None, None) == -1 and l.tbe_adamw_destroy(None) == 0


@pytest.mark.parametrize("buckets,far", [(1, 10), (2, 10), (16, 128), (32, 10 ** 7), (128, 200)])
def test_log_thresholds(buckets, far):
    from paper_2305_01515_amd.dense import log_thresholds
    t = log_thresholds(buckets, far)
    assert len(t) == buckets - 1 and all(b > a for a, b in zip([0] + t, t)) and all(x <= max(far, 2 * buckets) for x in t)


def test_adamw_counted():
    l, ptr = lib(), (C.c_void_p * 1)(16)
    assert l.tbe_adamw_step_counted(None, ptr, None, 0.0, 0.9, 0.9, 0.0, 0, None, None) == -1
    assert b"null handle" in l.tbe_last_error(None)
