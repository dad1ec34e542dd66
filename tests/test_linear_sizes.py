"""Sizes that 32 bits do not hold are refused, not cut to their low 32 bits (no GPU needed)."""
import ctypes

import pytest

from paper_2412_19867_b200 import binding as b

BIG = 2 ** 32


@pytest.fixture(scope="module", autouse=True)
def lib():
    from paper_2412_19867_b200 import build
    build.build()
    return b.load()


@pytest.mark.parametrize("C,K,gs", [(BIG + 64, 64, 32), (64, BIG + 64, 32), (64, 64, BIG + 32), (64, 64, -BIG + 32), (2 ** 31, 64, 32)])
def test_layer(C, K, gs):
    with pytest.raises(b.WfqError):
        b.wfq_linear_destroy(b.wfq_linear_create(C, K, gs))


def test_workspace():
    lin = b.wfq_linear_create(64, 64, 32)
    for call in (lambda: b.wfq_linear_workspace_bytes(lin, BIG + 1),
                 lambda: b.wfq_linear_set_workspace(lin, ctypes.c_void_p(4096), 1 << 40, BIG + 1)):
        with pytest.raises(b.WfqError):
            call()
    b.wfq_linear_destroy(lin)


@pytest.mark.parametrize("rows,C,gs", [(2, 64, BIG + 32), (2, 64, -BIG + 32), (2, BIG + 64, 0), (BIG + 2, 1, 32), (2, 64, 2 ** 63 - 1)])
def test_rows(rows, C, gs):
    """A group size of 2^32 + 32 would leave room for one scale per row and have two written."""
    with pytest.raises(b.WfqError):
        b.QuantizedRows(rows, C, gs, "meta")


def test_raw_calls():
    P = ctypes.c_void_p(4096)
    for sizes in ((BIG, 64, 32), (0, BIG + 64, 32), (0, 64, BIG + 32)):
        for call in (lambda: b.wfq_quantize_rows(P, 64, 0, *sizes, P, P), lambda: b.wfq_dequantize_rows(P, P, *sizes, 0, P, 64),
                     lambda: b.wfq_rms_norm_quantize(P, 64, None, 0, P, 1e-6, 0, *sizes, None, 0, P, P)):
            with pytest.raises(b.WfqError):
                call()
    lin = b.wfq_linear_create(64, 64, 32)
    for call in (lambda: b.wfq_linear_forward(lin, P, 64, BIG, None, 0, P, 64),
                 lambda: b.wfq_linear_forward_codes(lin, P, P, BIG, None, 0, P, 64)):
        with pytest.raises(b.WfqError) as err:
            call()
        assert err.value.status != b.WFQ_ERR_NOT_PREPARED
    b.wfq_linear_destroy(lin)


def test_rows_of_a_tensor():
    """More rows than 31 bits hold, in a tensor without memory."""
    class Tensor:
        is_cuda, shape = True, (BIG + 2, 1)

        def numel(self):
            return BIG + 2

        def is_contiguous(self):
            return True
    with pytest.raises(b.WfqError):
        b._rows_of(Tensor(), 1, "x")


@pytest.mark.parametrize("rows,C,gs", [(0, 64, 32), (3, 64, 2 ** 31 - 32), (2 ** 31 - 1, 1, 0)])
def test_sizes_that_fit(rows, C, gs):
    q = b.QuantizedRows(rows, C, gs, "meta")
    assert (q.rows, q.C, q.group_size) == (rows, C, gs)
