"""Row kernels whose CTAs go over the rows several times: the next row's loads under way, joined groups' maxima and the
row's sums in alternate halves of shared memory.  More rows than the SMs hold at once, in every way that a row is laid out."""
import pytest
import torch

from paper_2412_19867_b200 import binding as b
from tests import row_reference as ref

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.float16, torch.bfloat16]
# pieces of 8, 4 and single elements; groups within a warp's lanes, joined ones and whole rows; several rows a CTA (C < 500)
SHAPES = [(5003, 640, 64), (5003, 640, 96), (5003, 640, 0), (30011, 96, 32), (30011, 160, 96), (20011, 100, 32), (20011, 132, 96),
          (5003, 1500, 128), (5003, 1500, 96), (5003, 1500, 0), (4003, 1009, 32), (4003, 1009, 96), (4003, 1009, 0),
          (20011, 77, 32), (20011, 77, 0), (2003, 4096, 160), (1201, 9000, 96), (1201, 7777, 96), (1003, 20000, 0)]


def _rows(rows, C, dtype, seed):
    """Rows of sizes that differ from one to the next, so that a maximum or a sum left over from another row shows."""
    gen = torch.Generator(device="cuda").manual_seed(1000 * rows + C + seed)
    x = torch.randn((rows, C), generator=gen, device="cuda")
    return (x * torch.exp2(torch.randint(-6, 7, (rows, 1), generator=gen, device="cuda").float())).to(dtype)


def _check(q, codes, scales, rtol):
    rows, C = codes.shape
    got = q.codes.cpu()
    assert torch.equal(got[:, :C].double(), codes)
    assert not got[:, C:].any()
    s = q.scales[:, :rows].T.double().cpu()
    assert ((s - scales).abs() <= rtol * scales.abs() + 2.0 ** -149).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,C,gs", SHAPES)
def test_quantize(rows, C, gs, dtype):
    x = _rows(rows, C, dtype, 0)
    _check(b.quantize_rows(x, gs), *ref.quantize(x, gs), 0.0)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,C,gs", SHAPES)
def test_norm(rows, C, gs, dtype):
    x, res = _rows(rows, C, dtype, 0), _rows(rows, C, dtype, 1)
    gain = 1 + 0.3 * torch.randn(C, device="cuda", generator=torch.Generator("cuda").manual_seed(C))
    _, codes, scales = ref.rms_norm_quantize(x, None, gain, 1e-5, gs)
    _check(b.rms_norm_quantize(x, gain, 1e-5, gs)[0], codes, scales, ref.norm_scale_tolerance(C))
    want, codes, scales = ref.rms_norm_quantize(x, res, gain, 1e-5, gs)
    q, h = b.rms_norm_quantize(x, gain, 1e-5, gs, residual=res)
    assert torch.equal(h.cpu(), want)
    _check(q, codes, scales, ref.norm_scale_tolerance(C))
    q, h = b.rms_norm_quantize(x, gain, 1e-5, gs, residual=res, out=x)          # in place, rows asked ahead
    assert h is x and torch.equal(h.cpu(), want)
    _check(q, codes, scales, ref.norm_scale_tolerance(C))


@pytest.mark.parametrize("rows,C,gs", [(30011, 96, 32), (5003, 1500, 96), (4003, 1009, 96), (5003, 640, 64)])
def test_rows_that_are_not_finite_between_others(rows, C, gs):
    """Every third row holds a NaN, an infinity or nothing; the rows behind it are as they were."""
    x = _rows(rows, C, torch.bfloat16, 0)
    want = b.quantize_rows(x, gs)
    clean = want.codes.clone(), want.scales[:, :rows].clone()
    at = torch.arange(0, rows, 3, device="cuda")
    x[at[0::3], 5] = float("nan")
    x[at[1::3], C - 1] = float("inf")
    x[at[2::3]] = 0
    _check_other_rows = torch.ones(rows, dtype=torch.bool, device="cuda")
    _check_other_rows[at] = False
    q = b.quantize_rows(x, gs)
    assert torch.equal(q.codes[_check_other_rows], clean[0][_check_other_rows])
    assert torch.equal(q.scales[:, :rows][:, _check_other_rows], clean[1][:, _check_other_rows])
    codes, scales = ref.quantize(x, gs)
    assert torch.equal(q.codes[:, :C].cpu().double(), codes)
    assert torch.equal(torch.isnan(q.scales[:, :rows].T.cpu()), torch.isnan(scales))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,C,gs", [(30011, 96, 32), (20011, 77, 0), (20011, 132, 96), (3001, 2100, 64)])
def test_values_of_many_rows(rows, C, gs, dtype):
    q = b.quantize_rows(_rows(rows, C, torch.float32, 2), gs)
    want = q.codes[:, :C].cpu().double() * ref.spread(q.scales[:, :rows].T.double().cpu(), C, gs)
    v = b.dequantize_rows(q, dtype)
    half = torch.finfo(v.dtype).eps / 2
    assert ((v.double().cpu() - want).abs() <= half * want.abs() * (1 + 2.0 ** -12) + 2.0 ** -25).all()
