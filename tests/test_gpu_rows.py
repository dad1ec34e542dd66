"""Rows to codes and back, and the norm in front, against their definitions in 64 bits."""
import pytest
import torch

from paper_2412_19867_b200 import binding as b
from tests import row_reference as ref

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.float16, torch.bfloat16]


def _rows(rows, C, dtype, seed=0, size=1.0):
    gen = torch.Generator(device="cuda").manual_seed(1000 * rows + C + seed)
    x = torch.randn((rows, C), generator=gen, device="cuda") * size
    return torch.where(torch.rand((rows, C), generator=gen, device="cuda") < 0.02, 20.0 * x, x).to(dtype)


def _check(q, codes, scales, rtol):
    rows, C = codes.shape
    got = q.codes.cpu()
    assert torch.equal(got[:, :C].double(), codes)
    assert not got[:, C:].any()
    s = q.scales[:, :rows].T.double().cpu()
    nan = torch.isnan(scales)
    assert torch.equal(torch.isnan(s), nan)
    assert ((s - scales)[~nan].abs() <= rtol * scales[~nan].abs() + 2.0 ** -149).all()


SHAPES = [(1, 1, 32), (1, 4096, 128), (3, 31, 32), (5, 33, 32), (7, 64, 0), (129, 100, 64), (64, 160, 96), (33, 640, 64),
          (10, 1009, 32), (4, 1280, 256), (3, 1280, 512), (2, 5000, 0), (2, 8192, 128), (3, 16384, 32), (2, 20000, 160),
          (1, 40000, 128), (1, 131072, 0), (300, 136, 32), (260, 768, 32), (2, 2056, 64), (9, 24, 32), (1, 7, 0),
          (17, 1032, 96), (5, 12288, 4096)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,C,gs", SHAPES)
def test_quantize(rows, C, gs, dtype):
    x = _rows(rows, C, dtype)
    codes, scales = ref.quantize(x, gs)
    q = b.quantize_rows(x, gs)
    _check(q, codes, scales, 0.0)
    for name, t, half in (("f32", torch.float32, ref.U32), ("f16", torch.float16, 2.0 ** -11), ("bf16", torch.bfloat16, 2.0 ** -8)):
        v = b.dequantize_rows(q, name)
        want = codes * ref.spread(scales, C, gs)
        assert v.dtype is t and v.shape == x.shape
        assert ((v.double().cpu() - want).abs() <= half * want.abs() * (1 + 2.0 ** -12) + 2.0 ** -25).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("with_residual", [False, True])
@pytest.mark.parametrize("rows,C,gs", SHAPES)
def test_norm(rows, C, gs, with_residual, dtype):
    x, gain = _rows(rows, C, dtype), 1 + 0.3 * torch.randn(C, device="cuda", generator=torch.Generator("cuda").manual_seed(C))
    res = _rows(rows, C, dtype, 1) if with_residual else None
    h, codes, scales = ref.rms_norm_quantize(x, res, gain, 1e-5, gs)
    q, got_h = b.rms_norm_quantize(x, gain, 1e-5, gs, residual=res)
    _check(q, codes, scales, ref.norm_scale_tolerance(C))
    assert torch.equal(got_h.cpu(), h)


@pytest.mark.parametrize("where", ["new", "residual", "x"])
@pytest.mark.parametrize("C", [1009, 1280, 40000])
def test_stream_in_place(C, where):
    x, res = _rows(9, C, torch.bfloat16), _rows(9, C, torch.bfloat16, 1)
    gain = torch.ones(C, device="cuda")
    h, codes, scales = ref.rms_norm_quantize(x, res, gain, 1e-6, 64)
    out = {"new": None, "residual": res, "x": x}[where]
    q, got = b.rms_norm_quantize(x, gain, 1e-6, 64, residual=res, out=out)
    assert out is None or got is out
    assert torch.equal(got.cpu(), h)
    _check(q, codes, scales, ref.norm_scale_tolerance(C))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("C,ld,offset", [(640, 648, 0), (640, 641, 0), (640, 656, 3), (100, 100, 1), (64, 4096, 8)])
def test_strides_and_alignment(C, ld, offset, dtype):
    rows = 21
    flat = _rows(1, rows * ld + offset, dtype)[0]
    x = flat[offset:].as_strided((rows, C), (ld, 1))
    gain = torch.linspace(0.5, 2, C, device="cuda")
    codes, scales = ref.quantize(x, 64)
    _check(b.quantize_rows(x, 64), codes, scales, 0.0)
    out = torch.full((rows * ld + offset,), 7.0, dtype=dtype, device="cuda")
    view = out[offset:].as_strided((rows, C), (ld, 1))
    res = _rows(rows, C, dtype, 3)
    h, codes, scales = ref.rms_norm_quantize(x, res, gain, 1e-6, 64)
    q, got = b.rms_norm_quantize(x, gain, 1e-6, 64, residual=res, out=view)
    _check(q, codes, scales, ref.norm_scale_tolerance(C))
    assert torch.equal(got.cpu(), h)
    kept = torch.ones_like(out, dtype=torch.bool)
    kept[offset:].as_strided((rows, C), (ld, 1)).fill_(False)
    assert (out[kept] == 7.0).all()                                   # nothing beside the rows is written


@pytest.mark.parametrize("C,gs", [(256, 64), (1000, 96), (640, 0), (33, 32)])
def test_values_out_of_the_ordinary(C, gs):
    """Zeros, denormal groups, the largest finite values, infinities and NaN in single groups."""
    for dtype in TYPES:
        x = _rows(12, C, dtype)
        big = torch.finfo(dtype).max
        x[0] = 0
        x[1, :32] = 0
        x[2] = torch.finfo(dtype).tiny
        x[3, 5] = big
        x[4, 5] = -big
        x[5, 7] = float("inf")
        x[6, 7] = float("-inf")
        x[7, C - 1] = float("nan")
        x[8] = float("nan")
        x[9] = 1e-31 if dtype != torch.float16 else 0
        codes, scales = ref.quantize(x, gs)
        _check(b.quantize_rows(x, gs), codes, scales, 0.0)


def test_norm_of_rows_out_of_the_ordinary():
    C, gs = 256, 64
    x = _rows(6, C, torch.float32)
    x[0] = 0
    x[1, 3] = float("nan")                    # the whole row
    x[2, 3] = float("inf")                    # its group; the others are 0 times finite values
    x[3] *= 1e-12
    x[4] *= 1e12
    q, _ = b.rms_norm_quantize(x, torch.ones(C, device="cuda"), 1e-6, gs)
    s = q.scales[:, :6].T.cpu()
    assert (s[0] == 0).all() and torch.isnan(s[1]).all()
    assert torch.isnan(s[2, 0]) and (s[2, 1:] == 0).all()
    h, codes, scales = ref.rms_norm_quantize(x[3:], None, torch.ones(C), 1e-6, gs)
    assert torch.equal(q.codes[3:, :C].cpu().double(), codes)
    assert ((s[3:].double() - scales).abs() <= ref.norm_scale_tolerance(C) * scales.abs()).all()


def test_rows_behind_the_last_and_no_rows():
    C, gs, rows = 96, 32, 130
    x = _rows(rows, C, torch.float16)
    codes = torch.full((rows + 3, C), 55, dtype=torch.int8, device="cuda")
    scales = torch.full((3, 256), 9.0, device="cuda")
    stream = torch.cuda.current_stream().cuda_stream
    b.wfq_quantize_rows(x.data_ptr(), C, b.WFQ_F16, rows, C, gs, codes.data_ptr(), scales.data_ptr(), stream)
    torch.cuda.synchronize()
    assert (codes[rows:] == 55).all() and (scales[:, rows:] == 9.0).all() and not (scales[:, :rows] == 9.0).any()
    q = b.quantize_rows(x[:0], gs)
    assert q.rows == 0 and b.dequantize_rows(q).shape == (0, C)
    q, h = b.rms_norm_quantize(x[:0], torch.ones(C, device="cuda"), residual=x[:0])
    assert h.shape == (0, C)


def test_leading_dimensions_and_views():
    x = _rows(2 * 5 * 7, 64, torch.float16).reshape(2, 5, 7, 64)
    q = b.quantize_rows(x, 32)
    assert torch.equal(q.codes, b.quantize_rows(x.reshape(-1, 64), 32).codes) and b.dequantize_rows(q).shape == x.shape
    part = x[:, :, :, :32]                                           # rows at one distance of 64
    assert torch.equal(b.quantize_rows(part, 32).codes, b.quantize_rows(part.contiguous(), 32).codes)
    with pytest.raises(AssertionError):
        b.quantize_rows(x[:, :, 1:], 32)                             # two distances
    with pytest.raises(AssertionError):
        b.quantize_rows(x.transpose(2, 3), 32)


def test_offsets_beyond_32_bits():
    """A leading dimension that puts the last rows more than 2^32 bytes, and 2^31 elements, behind the first."""
    rows, C, ld = 5, 128, 600_000_000
    buf = torch.empty(ld * (rows - 1) + C, dtype=torch.float16, device="cuda")
    x = buf.as_strided((rows, C), (ld, 1))
    x.copy_(_rows(rows, C, torch.float16))
    codes, scales = ref.quantize(x, 64)
    q = b.quantize_rows(x, 64)
    _check(q, codes, scales, 0.0)
    h, codes, scales = ref.rms_norm_quantize(x, x, torch.ones(C), 1e-6, 64)
    q, got = b.rms_norm_quantize(x, torch.ones(C, device="cuda"), 1e-6, 64, residual=x, out=x)
    _check(q, codes, scales, ref.norm_scale_tolerance(C))
    assert torch.equal(got.cpu(), h)


def test_other_stream_and_graph():
    x, res = _rows(50, 640, torch.bfloat16), _rows(50, 640, torch.bfloat16, 1)
    gain = torch.ones(640, device="cuda")
    want, want_h = b.rms_norm_quantize(x, gain, residual=res)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got, got_h = b.rms_norm_quantize(x, gain, residual=res)
    side.synchronize()
    assert torch.equal(got.codes, want.codes) and torch.equal(got_h, want_h)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        q, h = b.rms_norm_quantize(x, gain, residual=res)
        v = b.dequantize_rows(q, "bf16")
    x.copy_(_rows(50, 640, torch.bfloat16, 5))
    graph.replay()
    want, want_h = b.rms_norm_quantize(x, gain, residual=res)
    assert torch.equal(q.codes, want.codes) and torch.equal(q.scales[:, :50], want.scales[:, :50])
    assert torch.equal(h, want_h) and torch.equal(v, b.dequantize_rows(want, "bf16"))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,C,gs", [(1, 4, 32), (3, 36, 32), (700, 100, 32), (601, 1500, 128), (5, 772, 0), (40, 4100, 160),
                                       (3, 12300, 64), (2, 20004, 256), (2, 131068, 0)])
def test_rows_in_pieces_of_four(rows, C, gs, dtype):
    """C a multiple of 4, not of 8: as they are, and inside wider rows that begin four elements in."""
    gain = torch.linspace(0.5, 2, C + 1, device="cuda")[1:]
    for ld, offset in ((C, 0), (C + 8, 4), (C + 4, 0)):
        x = _rows(1, rows * ld + offset, dtype, C)[0][offset:].as_strided((rows, C), (ld, 1))
        res = _rows(rows, C, dtype, 1)
        q = b.quantize_rows(x, gs)
        _check(q, *ref.quantize(x, gs), 0.0)
        h, codes, scales = ref.rms_norm_quantize(x, res, gain, 1e-5, gs)
        out = torch.full((rows * ld + offset,), 7.0, dtype=dtype, device="cuda")
        view = out[offset:].as_strided((rows, C), (ld, 1))
        qn, got = b.rms_norm_quantize(x, gain, 1e-5, gs, residual=res, out=view)
        _check(qn, codes, scales, ref.norm_scale_tolerance(C))
        assert torch.equal(got.cpu(), h)
        _, codes, scales = ref.rms_norm_quantize(x, None, gain, 1e-5, gs)
        _check(b.rms_norm_quantize(x, gain, 1e-5, gs)[0], codes, scales, ref.norm_scale_tolerance(C))
        name = {torch.float32: "f32", torch.float16: "f16", torch.bfloat16: "bf16"}[dtype]
        values = torch.full((rows * ld + offset,), 7.0, dtype=dtype, device="cuda")
        to = values[offset:].as_strided((rows, C), (ld, 1))
        b.wfq_dequantize_rows(q.codes.data_ptr(), q.scales.data_ptr(), rows, C, gs, b._DTYPES[name], to.data_ptr(), ld,
                              torch.cuda.current_stream().cuda_stream)
        assert torch.equal(to, b.dequantize_rows(q, name))
        want = q.codes[:, :C].double() * ref.spread(q.scales[:, :rows].T.double().cpu(), C, gs).cuda()
        half = torch.finfo(dtype).eps / 2
        assert ((to.double() - want).abs() <= half * want.abs() * (1 + 2.0 ** -12) + 2.0 ** -25).all()
        kept = torch.ones_like(out, dtype=torch.bool)
        kept[offset:].as_strided((rows, C), (ld, 1)).fill_(False)
        assert (out[kept] == 7.0).all() and (values[kept] == 7.0).all()
