"""Activations of the linear layer where their argument is out of the ordinary, on every path to the output."""
import pytest
import torch

from paper_2412_19867_b200 import binding as b

pytestmark = pytest.mark.gpu

NAMES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
ACTS = {"none": b.WFQ_ACT_NONE, "relu": b.WFQ_ACT_RELU, "silu": b.WFQ_ACT_SILU, "gelu": b.WFQ_ACT_GELU}
# dot products; outputs on the lanes; rows on the lanes; pairs; channels shared by a cluster in both orientations
SHAPES = [14004, 12016, 12064, 11064, 11128, 13128, 13256, 22032, 41064]


def _rand(shape, dtype, seed, size=1.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=gen, device="cuda") * size).to(dtype)


def _layer(w, gs, rows, dtype, shape, bias, act, gated, out=None):
    layer = b.Linear(w.shape[1], w.shape[0] // (2 if gated else 1), gs, rows, dtype, out_dtype=out, gated=gated)
    layer.prepare(w)
    layer.set_epilogue(bias, ACTS[act])
    b.wfq_linear_set_debug_option(layer.lin, b.WFQ_DEBUG_GEMM_SHAPE, shape)
    return layer


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("act", list(ACTS))
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("K,dtype", [(96, "bf16"), (75, "f32"), (128, "f16")])       # wide stores and single ones
def test_rows_that_are_not_finite_stay_so(K, dtype, gated, act, shape):
    t, rows, C = NAMES[dtype], 7 if shape == 14004 else 300, 1024
    w = _rand(((2 if gated else 1) * K, C), t, 1, C ** -0.5)
    bias, res, x = _rand((len(w),), torch.float32, 2), _rand((rows, K), t, 3), _rand((rows, C), t, 4)
    layer = _layer(w, 128, rows, dtype, shape, bias, act, gated)
    clean = layer.forward(x, residual=res)
    assert torch.isfinite(clean).all()
    x[1, 100] = float("nan")
    x[2, 5] = float("inf")
    x[rows - 1, C - 1] = float("-inf")
    bad = torch.zeros(rows, dtype=torch.bool, device="cuda")
    bad[[1, 2, rows - 1]] = True
    for y in (layer.forward(x, residual=res), layer.forward_codes(b.quantize_rows(x, 128), residual=res)):
        assert torch.isnan(y[bad]).all()
        assert torch.equal(y[~bad], clean[~bad])
    layer.check_status()


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("act", list(ACTS))
@pytest.mark.parametrize("gated", [False, True])
def test_weights_and_bias_that_are_not_finite(gated, act, shape):
    """They reach their own column and no other."""
    rows, C, K = 7 if shape == 14004 else 200, 1024, 96
    w, x = _rand(((2 if gated else 1) * K, C), torch.float32, 1, C ** -0.5), _rand((rows, C), torch.float32, 4)
    bias = _rand((len(w),), torch.float32, 2)
    clean = _layer(w, 128, rows, "f32", shape, bias, act, gated).forward(x)
    assert torch.isfinite(clean).all()
    w[7, 300] = float("nan")
    w[40, 1] = float("inf")
    bias[11] = float("nan")
    layer = _layer(w, 128, rows, "f32", shape, bias, act, gated)
    y = layer.forward(x)
    bad = torch.zeros(K, dtype=torch.bool, device="cuda")
    bad[[7, 40, 11]] = True
    assert torch.isnan(y[:, bad]).all()
    assert torch.equal(y[:, ~bad], clean[:, ~bad])
    layer.check_status()
