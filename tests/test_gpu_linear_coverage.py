"""The linear layer where the other tests do not reach: warps of the dot products that go on to further columns, residuals
in place over many tiles, outputs far apart in memory."""
import pytest
import torch

from paper_2412_19867_b200 import binding as b
from tests import row_reference as ref

pytestmark = pytest.mark.gpu

NAMES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def _rand(shape, dtype, seed, size=1.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=gen, device="cuda") * size).to(NAMES[dtype])


def _layer(C, K, gs, rows, dtype, seed=1, gated=False, shape=0):
    layer = b.Linear(C, K, gs, rows, dtype, gated=gated)
    w = _rand(((2 if gated else 1) * K, C), dtype, seed, C ** -0.5)
    layer.prepare(w)
    if shape:
        b.wfq_linear_set_debug_option(layer.lin, b.WFQ_DEBUG_GEMM_SHAPE, shape)
    return layer, w


@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("rows", [1, 2, 3, 5, 8])
@pytest.mark.parametrize("C,gs,dtype", [(64, 32, "f16"), (200, 64, "f32"), (500, 0, "bf16"), (1600, 96, "bf16"), (2100, 128, "f16")])
def test_dot_products_over_many_columns(C, gs, dtype, rows, gated, codes):
    """20001 columns (or 2 x 10001) are more than all warps have at a time; 2100 channels are more than one turn of a warp."""
    K = 10001 if gated else 20001
    layer, w = _layer(C, K, gs, rows, dtype, gated=gated, shape=14004)
    bias = _rand((len(w),), "f32", 5, 0.5)
    layer.set_epilogue(bias, b.WFQ_ACT_SILU)
    x, res = _rand((rows, C), dtype, 2), _rand((rows, K), dtype, 3)
    y = layer.forward_codes(b.quantize_rows(x, gs), residual=res) if codes else layer.forward(x, residual=res)
    want, tol = ref.linear(*ref.quantize(x, gs), *ref.quantize(w, gs), gs, bias, "silu", gated, res, NAMES[dtype])
    off = (y.double().cpu() - want).abs()
    assert (off <= tol).all(), (float((off / tol).max()), int((off > tol).sum()))
    layer.close()


@pytest.mark.parametrize("shape", [11064, 11128, 12016, 12032, 12064, 13128, 13256])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("ld", [2056, 2059])
def test_residual_in_place_over_many_tiles(ld, dtype, gated, shape):
    """Residuals are asked for up to 64 columns ahead of the outputs that take their place."""
    rows, C, K = 1300, 160, 2056
    layer, _ = _layer(C, K, 64, rows, dtype, gated=gated, shape=shape)
    layer.set_epilogue(None, b.WFQ_ACT_SILU)
    x, res = _rand((rows, C), dtype, 2), _rand((rows, K), dtype, 3)
    want = layer.forward(x, residual=res)
    flat = torch.full((rows, ld), 7.0, dtype=NAMES[dtype], device="cuda")
    y = flat[:, :K]
    for _ in range(3):
        y.copy_(res)
        layer.forward(x, residual=y, y=y)
        assert torch.equal(y, want)
    assert (flat[:, K:] == 7.0).all()
    layer.check_status()


@pytest.mark.parametrize("shape,rows", [(14004, 5), (14004, 8), (12016, 9), (12064, 40), (11064, 40), (11128, 40), (13128, 40), (13256, 40),
                                        (22016, 9), (41064, 40)])
@pytest.mark.parametrize("aligned", [True, False])
def test_offsets_beyond_32_bits(shape, rows, aligned):
    """Rows of y and of the residual that lie more than 2^32 elements behind the first, and x likewise."""
    C, K = 512, 136
    ld = (4_400_000_000 // (rows - 1) + 7) // 8 * 8 + (0 if aligned else 1)
    layer, _ = _layer(C, K, 128, rows, "f16", shape=shape)
    x, res = _rand((rows, C), "f16", 2), _rand((rows, K), "f16", 3)
    want = layer.forward(x, residual=res)
    buf = torch.empty(ld * (rows - 1) + 2048, dtype=torch.float16, device="cuda")
    xv, yv = buf.as_strided((rows, C), (ld, 1)), buf[1024:].as_strided((rows, K), (ld, 1))
    for r in range(rows):
        buf[r * ld:r * ld + 2048] = 7.0 if r * ld + 2048 <= len(buf) else 0.0
    xv.copy_(x)
    yv.copy_(res)
    layer.forward(xv, residual=yv, y=yv)
    assert torch.equal(yv, want)
    assert torch.equal(xv, x) and (buf[:1024][C:] == 7.0).all() and (buf[1024 + K:2048] == 7.0).all()
    layer.check_status()
    del buf


def test_weights_far_apart():
    """A leading dimension of the weights that puts the last ones more than 2^32 elements behind the first."""
    K, C, ld = 9, 96, 600_000_000
    w = _rand((K, C), "f16", 1, C ** -0.5)
    buf = torch.empty(ld * (K - 1) + C, dtype=torch.float16, device="cuda")
    far = buf.as_strided((K, C), (ld, 1))
    far.copy_(w)
    x = _rand((4, C), "f16", 2)
    near, other = b.Linear(C, K, 32, 4, "f16"), b.Linear(C, K, 32, 4, "f16")
    near.prepare(w)
    other.prepare(far)
    assert torch.equal(near.forward(x), other.forward(x))


@pytest.mark.parametrize("large", ["x", "w"])
@pytest.mark.parametrize("shape,rows", [(14004, 3), (12016, 9), (12064, 40), (11064, 40), (11128, 200), (13128, 40), (13256, 300), (22032, 9)])
@pytest.mark.parametrize("C,gs", [(256, 128), (1024, 0)])
def test_largest_values(C, gs, shape, rows, large):
    """All codes 127 and values at 0.95 of the range that the header gives: the scaled sum of a group is just below 3.4e38."""
    K, a, c = 70, 0.95 * 2.68e36 / (gs or C), 1e-28
    x = torch.full((rows, C), a if large == "x" else c, device="cuda")
    w = torch.full((K, C), c if large == "x" else a, device="cuda")
    layer = b.Linear(C, K, gs, rows, "f32")
    layer.prepare(w)
    b.wfq_linear_set_debug_option(layer.lin, b.WFQ_DEBUG_GEMM_SHAPE, shape)
    want, tol = ref.linear(*ref.quantize(x, gs), *ref.quantize(w, gs), gs)
    for y in (layer.forward(x), layer.forward_codes(b.quantize_rows(x, gs))):
        assert ((y.double().cpu() - want).abs() <= tol).all()


@pytest.mark.parametrize("rows,C,K,parts", [(40_000, 65_536, 48, "x"), (70_000, 64, 32_768, "y"), (300, 1024, 2_200_000, "w"),
                                            (2, 1024, 2_200_000, "w"), (20, 1024, 2_200_000, "w")])
def test_more_than_2_to_31_elements(rows, C, K, parts):
    """Codes of x, y or codes of the weights beyond 2^31 (the residual in place with y): the last rows and columns against a
    layer of their own."""
    gs = 128
    layer = b.Linear(C, K, gs, rows, "bf16")
    x = torch.randn((rows, C), device="cuda", generator=torch.Generator("cuda").manual_seed(1), dtype=torch.bfloat16)
    w = torch.randn((K, C), device="cuda", generator=torch.Generator("cuda").manual_seed(2), dtype=torch.bfloat16)
    y = torch.empty((rows, K), dtype=torch.bfloat16, device="cuda")
    for i in range(0, rows, 4096):
        y[i:i + 4096] = (torch.arange(K, device="cuda") % 13 - 6).bfloat16()
    layer.prepare(w)
    layer.forward(x, residual=y, y=y)
    layer.check_status()
    r, k = min(rows, 130), min(K, 140)
    for rs in (slice(0, r), slice(rows - r, rows)):
        for ks in (slice(0, k), slice(K - k, K)):
            res = (torch.arange(K, device="cuda")[ks] % 13 - 6).bfloat16().expand(r, k).contiguous()
            want, tol = ref.linear(*ref.quantize(x[rs], gs), *ref.quantize(w[ks], gs), gs, residual=res, dtype=torch.bfloat16)
            assert ((y[rs, ks].double().cpu() - want).abs() <= tol).all()
