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


def _normal_cdf_times(t):
    """t Phi(t) in 64 bits without cancellation."""
    return 0.5 * t * torch.special.erfc(-t * 0.5 ** 0.5)


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("gated", [False, True])
def test_gelu_over_its_range(gated, shape):
    """Rows of zeros: the outputs are the activation of the bias, gated times the other half's bias.

    Bound in units of 2^-23, with Phi(-a) = exp(-a^2 / 2) s P(s), s = 1 / (1 + 0.3 a): the exponent's two products and its
    constant 3 / 2 units of a^2 / 2 = 0.75 t^2; the exponential 2; s 1.5 (sum, reciprocal) times the slope
    |d ln(s P) / d ln s| <= 2.7: 4; the polynomial's seven steps half a unit of each partial value, 1.6 of the result, its
    rounded coefficients 1, its fit 1.1; three products 1.5: in all 11.2 + 0.75 t^2.  For t > 0 that is an error of q <= 1 / 2
    in 1 - q >= 1 / 2, and two roundings: 12.2.  The gate's product half a unit, the rest for what is of second order.  An
    exponential below 2^-126 is 0: an error of 2^-127 |t|, times the gate's other half; no number is finer than 2^-149."""
    t = torch.cat([torch.linspace(-14, 14, 1401), torch.logspace(-38, 38, 300), -torch.logspace(-38, 38, 300),
                   torch.tensor([0.0, float("inf")])]).float().cuda()
    K, rows = len(t), 5 if shape == 14004 else 150
    value = 10.0 ** torch.linspace(-3, 3, K, device="cuda")[torch.randperm(K, generator=torch.Generator("cuda").manual_seed(1), device="cuda")]
    w = torch.zeros(((2 if gated else 1) * K, 1024), device="cuda")
    layer = _layer(w, 128, rows, "f32", shape, torch.cat([t, value]) if gated else t, "gelu", gated)
    y = layer.forward(torch.zeros((rows, 1024), device="cuda"))
    assert torch.equal(y, y[:1].expand_as(y))
    got, x, v = y[0].double(), t.double(), value.double() if gated else torch.ones(K, device="cuda", dtype=torch.float64)
    want = _normal_cdf_times(x) * v
    finite = torch.isfinite(want) & (want.abs() < 3.4e38)
    bound = (13 + 0.75 * x.clamp(-20, 0) ** 2) * 2.0 ** -23 * want.abs() + 2.0 ** -126 * x.abs() * v + 2.0 ** -149 * (v + 1)
    off = (got - want).abs()
    assert (off <= bound)[finite].all(), float((off / bound)[finite].max())
    assert got[-1] == float("inf")
