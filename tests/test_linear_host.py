"""Refusals of the row operators and the linear layer, all before any device work (no GPU needed)."""
import ctypes

import pytest

from paper_2412_19867_b200 import binding as b

P = ctypes.c_void_p(4096)                  # aligned, never read: every call here is refused or has no rows
INVALID, UNSUPPORTED, OK = b.WFQ_ERR_INVALID_ARG, b.WFQ_ERR_UNSUPPORTED, b.WFQ_OK


@pytest.fixture(scope="module")
def lib():
    from paper_2412_19867_b200 import build
    build.build()
    return b.load()


def _with(base, **change):
    args = dict(base, **change)
    return list(args.values())


NORM = dict(x=P, ldx=64, res=P, ldr=64, gain=P, eps=1e-6, dtype=b.WFQ_F16, rows=2, C=64, gs=32, h=P, ldh=64, codes=P,
            scales=P, stream=None)


@pytest.mark.parametrize("change,status", [
    (dict(x=None), INVALID), (dict(gain=None), INVALID), (dict(codes=None), INVALID), (dict(scales=None), INVALID),
    (dict(ldx=63), INVALID), (dict(ldr=63), INVALID), (dict(ldh=0), INVALID), (dict(rows=-1), INVALID), (dict(C=0), INVALID),
    (dict(gs=-32), INVALID), (dict(gs=33), UNSUPPORTED), (dict(gs=16), UNSUPPORTED), (dict(C=131073, ldx=1 << 20), UNSUPPORTED),
    (dict(rows=0x7fffff01), UNSUPPORTED), (dict(dtype=3), INVALID), (dict(dtype=-1), INVALID), (dict(eps=-1e-6), INVALID),
    (dict(eps=float("nan")), INVALID), (dict(eps=float("inf")), INVALID), (dict(res=None), INVALID),
    (dict(x=ctypes.c_void_p(4097)), INVALID), (dict(res=ctypes.c_void_p(4097)), INVALID), (dict(h=ctypes.c_void_p(4097)), INVALID),
    (dict(gain=ctypes.c_void_p(4098)), INVALID), (dict(codes=ctypes.c_void_p(4096 + 16)), INVALID),
    (dict(scales=ctypes.c_void_p(4096 + 8)), INVALID), (dict(dtype=b.WFQ_F32, x=ctypes.c_void_p(4098)), INVALID),
    (dict(rows=0), OK), (dict(rows=0, x=None, codes=None), OK)])
def test_norm(lib, change, status):
    assert lib.wfq_rms_norm_quantize(*_with(NORM, **change)) == status


@pytest.mark.parametrize("change,status", [
    (dict(x=None), INVALID), (dict(ldx=63), INVALID), (dict(dtype=9), INVALID), (dict(rows=-5), INVALID), (dict(C=-1), INVALID),
    (dict(gs=100), UNSUPPORTED), (dict(codes=None), INVALID), (dict(scales=None), INVALID),
    (dict(codes=ctypes.c_void_p(4096 + 8)), INVALID), (dict(scales=ctypes.c_void_p(4100)), INVALID), (dict(rows=0), OK)])
def test_quantize(lib, change, status):
    base = dict(x=P, ldx=64, dtype=b.WFQ_BF16, rows=2, C=64, gs=32, codes=P, scales=P, stream=None)
    assert lib.wfq_quantize_rows(*_with(base, **change)) == status


@pytest.mark.parametrize("change,status", [
    (dict(codes=None), INVALID), (dict(scales=None), INVALID), (dict(v=None), INVALID), (dict(ldv=63), INVALID),
    (dict(dtype=4), INVALID), (dict(gs=48), UNSUPPORTED), (dict(rows=-1), INVALID), (dict(v=ctypes.c_void_p(4097)), INVALID),
    (dict(rows=0), OK)])
def test_dequantize(lib, change, status):
    base = dict(codes=P, scales=P, rows=2, C=64, gs=32, dtype=b.WFQ_F16, v=P, ldv=64, stream=None)
    assert lib.wfq_dequantize_rows(*_with(base, **change)) == status


def _create(lib, *args):
    lin = ctypes.c_void_p()
    return lib.wfq_linear_create(ctypes.byref(lin), *args), lin


def test_create(lib):
    assert lib.wfq_linear_create(None, 64, 64, 32, 0) == INVALID
    for args, want in {(0, 64, 32, 0): INVALID, (64, 0, 32, 0): INVALID, (64, 64, -32, 0): INVALID, (64, 64, 32, 2): INVALID,
                       (64, 64, 32, -1): INVALID, (64, 64, 40, 0): UNSUPPORTED, (131073, 64, 32, 0): UNSUPPORTED,
                       (64, (1 << 22) + 1, 32, 0): UNSUPPORTED}.items():
        st, lin = _create(lib, *args)
        assert st == want and not lin.value, args
    for args in ((1, 1, 0, 0), (64, 64, 32, 1), (131072, 1 << 22, 0, 1), (100, 7, 64, 0), (64, 64, 4096, 0)):
        st, lin = _create(lib, *args)
        assert st == OK and lin.value
        assert lib.wfq_linear_destroy(lin) == OK
    assert lib.wfq_linear_destroy(None) == OK


def test_workspace_and_order_of_calls(lib):
    st, lin = _create(lib, 100, 96, 64, 0)                     # 128 codes a row, two groups
    up = lambda v: (v + 1023) // 1024 * 1024
    for rows in (1, 8, 129, 5000):
        assert lib.wfq_linear_workspace_bytes(lin, rows) == up(rows * 128) + up(2 * ((rows + 127) // 128 * 128) * 4)
    assert lib.wfq_linear_workspace_bytes(None, 1) == 0 and lib.wfq_linear_workspace_bytes(lin, 0) == 0
    n = lib.wfq_linear_workspace_bytes(lin, 8)
    for ptr, size, rows in ((None, n, 8), (P, n - 1, 8), (ctypes.c_void_p(4096 + 512), n, 8), (P, n, 0), (P, n, 16)):
        if rows == 16 and lib.wfq_linear_workspace_bytes(lin, 16) == n:
            continue
        assert lib.wfq_linear_set_workspace(lin, ptr, size, rows) == INVALID
    assert lib.wfq_linear_forward(lin, P, 100, 1, None, 0, P, 96, None) == b.WFQ_ERR_NOT_PREPARED
    assert lib.wfq_linear_forward_codes(lin, P, P, 1, None, 0, P, 96, None) == b.WFQ_ERR_NOT_PREPARED
    assert lib.wfq_linear_check_status(lin, None, None) == b.WFQ_ERR_NOT_PREPARED
    ptr, size = ctypes.c_void_p(), ctypes.c_size_t()
    assert lib.wfq_linear_debug_get(lin, b.WFQ_BUF_WQ, ctypes.byref(ptr), ctypes.byref(size)) == b.WFQ_ERR_NOT_PREPARED
    assert lib.wfq_linear_debug_get(lin, b.WFQ_BUF_Y, ctypes.byref(ptr), ctypes.byref(size)) == INVALID
    assert lib.wfq_linear_forward(lin, P, 100, -1, None, 0, P, 96, None) == INVALID
    for args in ((None, 100, b.WFQ_F16), (P, 99, b.WFQ_F16), (P, 100, 5), (ctypes.c_void_p(4097), 100, b.WFQ_F16),
                 (ctypes.c_void_p(4098), 100, b.WFQ_F32)):
        assert lib.wfq_linear_prepare_weights(lin, *args, None) == INVALID
    lib.wfq_linear_destroy(lin)


def test_settings(lib):
    st, lin = _create(lib, 512, 96, 64, 0)
    for dt in (b.WFQ_F32, b.WFQ_F16, b.WFQ_BF16):
        assert lib.wfq_linear_set_input_dtype(lin, dt) == OK and lib.wfq_linear_set_output_dtype(lin, dt) == OK
    assert lib.wfq_linear_set_input_dtype(lin, 3) == INVALID and lib.wfq_linear_set_output_dtype(lin, -1) == INVALID
    for act in range(4):
        assert lib.wfq_linear_set_epilogue(lin, None, act) == OK
    assert lib.wfq_linear_set_epilogue(lin, None, 4) == INVALID and lib.wfq_linear_set_epilogue(lin, None, -1) == INVALID
    assert lib.wfq_linear_set_epilogue(lin, ctypes.c_void_p(4097), 0) == INVALID
    ll = ctypes.c_longlong
    for value, want in ((0, OK), (11064, OK), (41128, OK), (42016, OK), (13256, OK), (23256, INVALID), (11256, INVALID), (82016, INVALID), (31064, INVALID), (11032, INVALID),
                        (12128, INVALID), (13064, INVALID), (14064, INVALID), (14004, OK), (24004, INVALID), (111064, INVALID), (1064, INVALID), (-11064, INVALID)):
        assert lib.wfq_linear_set_debug_option(lin, b.WFQ_DEBUG_GEMM_SHAPE, ll(value)) == want, value
    assert lib.wfq_linear_set_debug_option(lin, b.WFQ_DEBUG_WAIT_CYCLES, ll(999)) == INVALID
    assert lib.wfq_linear_set_debug_option(lin, b.WFQ_DEBUG_SKIP_GEMM_STAGE, ll(-2)) == INVALID
    assert lib.wfq_linear_set_debug_option(lin, b.WFQ_DEBUG_GEMM_CTAS, ll(1)) == INVALID
    lib.wfq_linear_destroy(lin)


def test_null_layer(lib):
    assert lib.wfq_linear_set_input_dtype(None, 0) == INVALID and lib.wfq_linear_set_output_dtype(None, 0) == INVALID
    assert lib.wfq_linear_set_epilogue(None, None, 0) == INVALID
    assert lib.wfq_linear_set_workspace(None, P, 1 << 30, 1) == INVALID
    assert lib.wfq_linear_prepare_weights(None, P, 64, 0, None) == INVALID
    assert lib.wfq_linear_forward(None, P, 64, 1, None, 0, P, 64, None) == INVALID
    assert lib.wfq_linear_forward_codes(None, P, P, 1, None, 0, P, 64, None) == INVALID
    assert lib.wfq_linear_set_debug_option(None, b.WFQ_DEBUG_WAIT_CYCLES, ctypes.c_longlong(5000)) == INVALID
    assert lib.wfq_linear_check_status(None, None, None) == INVALID


def test_gelu_is_no_activation_of_the_convolution(lib):
    plan = b.wfq_plan_create(1, 64, 64, 8, 8, 4, 3, 32, 8)
    assert lib.wfq_plan_set_epilogue(plan, None, b.WFQ_ACT_GELU) == INVALID
    b.wfq_plan_destroy(plan)
