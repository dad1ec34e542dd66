"""What may lie in place and what is refused: a result that lands on another row's input, or on the input of a product."""
import ctypes

import pytest

from paper_2412_19867_b200 import binding as b

P, Q, R = ctypes.c_void_p(4096), ctypes.c_void_p(8192), ctypes.c_void_p(1 << 20)       # never read


@pytest.mark.parametrize("rows,x,ldx,res,ldr,h,ldh", [(2, P, 64, Q, 64, P, 128), (2, P, 128, Q, 64, P, 64),
                                                      (5, P, 64, Q, 64, Q, 72), (5, P, 64, P, 80, P, 64), (2, P, 64, P, 64, P, 65)])
def test_norm_onto_other_rows_is_refused(rows, x, ldx, res, ldr, h, ldh):
    from paper_2412_19867_b200 import build
    build.build()
    lib = b.load()
    assert lib.wfq_rms_norm_quantize(x, ldx, res, ldr, R, 1e-6, b.WFQ_F16, rows, 64, 32, h, ldh, R, R, None) == b.WFQ_ERR_INVALID_ARG


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [1, 4, 40, 300])
def test_product(rows):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(rows)
    x = torch.randn((rows, 256), generator=gen, device="cuda").half()
    layer = b.Linear(256, 256, 64, rows, "f16")
    layer.prepare(torch.randn((256, 256), generator=gen, device="cuda").half())
    want = layer.forward(x, residual=x)
    wide = torch.zeros((rows, 600), dtype=torch.float16, device="cuda")
    wide[:, :256], wide[:, 300:556] = x, x
    kept = wide.clone()
    with pytest.raises(b.WfqError):
        layer.forward(x, residual=x, y=x)
    with pytest.raises(b.WfqError):
        layer.forward(wide[:, :256], y=wide[:, :256])
    y = x.clone()
    layer.forward(x, residual=y, y=y)                              # the residual in place
    assert torch.equal(y, want)
    layer.forward(wide[:, :256], residual=wide[:, 300:556], y=wide[:, 300:556])       # beside the input
    assert torch.equal(wide[:, 300:556], want)
    wide[:, 300:556] = x
    assert torch.equal(wide, kept)
    if rows > 1:
        flat = torch.zeros(rows * 300, dtype=torch.float16, device="cuda")
        with pytest.raises(b.WfqError):
            layer.forward(x, residual=flat[:rows * 256].view(rows, 256), y=flat.view(rows, 300)[:, :256])
    q = b.quantize_rows(x, 64)
    stream = torch.cuda.current_stream().cuda_stream
    with pytest.raises(b.WfqError):
        b.wfq_linear_forward_codes(layer.lin, q._codes, q._scales, rows, None, 0, q._codes, 256, stream)
    with pytest.raises(b.WfqError):
        b.wfq_linear_forward(layer.lin, x.data_ptr(), 256, rows, None, 0, x.data_ptr(), 256, stream)
    y = torch.empty_like(x)
    b.wfq_linear_forward(layer.lin, x.data_ptr(), 256, rows, x.data_ptr(), 256, y.data_ptr(), 256, stream)
    assert torch.equal(y, want)
    y = torch.empty_like(x)
    b.wfq_linear_forward_codes(layer.lin, q._codes, q._scales, rows, x.data_ptr(), 256, y.data_ptr(), 256, stream)
    assert torch.equal(y, want)
    layer.check_status()


@pytest.mark.gpu
@pytest.mark.parametrize("C", [96, 1009, 40000])
def test_norm_without_its_stream(C):
    """The sum is formed for the norm alone where no one asks for it."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(C)
    x, res = (torch.randn((11, C), generator=gen, device="cuda").bfloat16() for _ in range(2))
    gain = torch.rand(C, generator=gen, device="cuda") + 0.5
    want, _ = b.rms_norm_quantize(x, gain, 1e-6, 64, residual=res)
    q = b.QuantizedRows(11, C, 64, "cuda")
    kept = x.clone(), res.clone()
    b.wfq_rms_norm_quantize(x.data_ptr(), C, res.data_ptr(), C, gain.data_ptr(), 1e-6, b.WFQ_BF16, 11, C, 64, None, 0,
                            q._codes, q._scales, torch.cuda.current_stream().cuda_stream)
    assert torch.equal(q.codes, want.codes) and torch.equal(q.scales[:, :11], want.scales[:, :11])
    assert torch.equal(x, kept[0]) and torch.equal(res, kept[1])
