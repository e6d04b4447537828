"""Arguments that the C entry points of the norm, the short convolution and the selective scan refuse before they touch a GPU."""
import ctypes as C


def lib():
    from paper_2305_01515_amd import dense
    return dense._lib()


def test_norm():
    from paper_2305_01515_amd.dense import NormBatch, NormGrad
    l, h, nan = lib(), C.c_void_p(), float("nan")
    for dim, dtype, residual, eps, rows, code in ((0, 0, -1, 0.0, 1, -1), (32769, 0, -1, 0.0, 1, -1), (8, 3, -1, 0.0, 1, -1), (8, 0, 1, 0.0, 1, -1), (8, 1, 2, 0.0, 1, -1),
                                                  (8, 0, -2, 0.0, 1, -1), (8, 0, 0, -1e-9, 1, -1), (8, 0, 0, nan, 1, -1), (8, 0, 0, 0.0, -1, -1), (32768, 0, 0, 0.0, 1 << 40, -5)):
        assert l.tbe_norm_create(C.byref(h), dim, dtype, residual, eps, rows) == code and not h
    assert l.tbe_norm_create(None, 8, 0, -1, 0.0, 1) == -1 and l.tbe_norm_destroy(None) == 0
    b, g = NormBatch(), NormGrad()
    assert l.tbe_norm_forward(None, C.byref(b), None, 8, None, None) == -1 and l.tbe_norm_forward(None, None, None, 8, None, None) == -1
    assert l.tbe_norm_backward(None, C.byref(g), None) == -1 and l.tbe_norm_backward(None, None, None) == -1
    for group in (8, 24, 512, -1):
        assert l.tbe_norm_quantise(None, C.byref(b), group, None, 8, None, None) == -1
        assert b"power of two" in l.tbe_last_error(None)


def test_conv():
    from paper_2305_01515_amd.dense import ConvBatch
    l, h = lib(), C.c_void_p()
    for dim, width, dtype, bags, rows, code in ((0, 4, 0, 1, 1, -1), (65537, 4, 0, 1, 1, -1), (8, 0, 0, 1, 1, -1), (8, 9, 0, 1, 1, -1), (8, 4, 3, 1, 1, -1), (8, 4, 0, -1, 1, -1),
                                                (8, 4, 0, 1, -1, -1), (65536, 4, 0, 1, 1 << 40, -5), (8, 4, 0, 1 << 31, 1, -5)):
        assert l.tbe_conv_create(C.byref(h), dim, width, dtype, 1, bags, rows) == code and not h
    b = ConvBatch()
    assert l.tbe_conv_create(None, 8, 4, 0, 1, 1, 1) == -1 and l.tbe_conv_destroy(None) == 0 and l.tbe_conv_check(None, None) == -1
    assert l.tbe_conv_forward(None, C.byref(b), None, 8, None, None) == -1
    assert l.tbe_conv_backward(None, C.byref(b), None, 8, None, None, 8, None, None, None, None) == -1
    assert l.tbe_conv_step(None, C.byref(b), None, 1, None, None, 8, None) == -1
    assert b"null handle" in l.tbe_last_error(None)


def test_ssm():
    from paper_2305_01515_amd.dense import SsmBatch, SsmGrads
    l, h = lib(), C.c_void_p()
    for dim, states, groups, dtype, bags, rows, code in ((0, 16, 1, 0, 1, 1, -1), (65537, 16, 1, 0, 1, 1, -1), (8, 0, 1, 0, 1, 1, -1), (8, 65, 1, 0, 1, 1, -1), (64, 16, 2, 0, 1, 1, -1),
                                                         (130, 16, 2, 0, 1, 1, -1), (8, 16, 0, 0, 1, 1, -1), (8, 16, 1, 3, 1, 1, -1), (8, 16, 1, 0, -1, 1, -1), (8, 16, 1, 0, 1, -1, -1),
                                                         (65536, 16, 1, 0, 1, 1 << 40, -5), (65536, 64, 1, 0, 1 << 30, 1, -5)):
        assert l.tbe_ssm_create(C.byref(h), dim, states, groups, dtype, bags, rows) == code and not h
    b, g = SsmBatch(), SsmGrads()
    assert l.tbe_ssm_create(None, 8, 16, 1, 0, 1, 1) == -1 and l.tbe_ssm_destroy(None) == 0 and l.tbe_ssm_check(None, None) == -1
    assert l.tbe_ssm_forward(None, C.byref(b), None, 8, None, None, None) == -1 and l.tbe_ssm_saved_floats(None, 1) == -1
    assert l.tbe_ssm_backward(None, C.byref(b), None, C.byref(g), None) == -1
    assert l.tbe_ssm_step(None, C.byref(b), None, 8, 1, None, None, 8, None) == -1
    assert b"null handle" in l.tbe_last_error(None)


def test_ssm_grids():
    """rows and bags whose units and offsets would take a launch of 2^32 lanes"""
    l, h = lib(), C.c_void_p()
    for dim, bags, rows in ((1, 1, 67108863 * 128), (1, 1 << 30, 60 * (1 << 20) * 128), (64, (1 << 31) - 2, 1 << 32)):
        assert l.tbe_ssm_create(C.byref(h), dim, 1, 1, 0, bags, rows) == -5 and not h
