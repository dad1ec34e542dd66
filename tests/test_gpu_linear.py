"""The linear layer against its definition in 64 bits: every kernel shape, type, epilogue, width and stride."""
import pytest
import torch

from paper_2412_19867_b200 import binding as b
from tests import row_reference as ref

pytestmark = pytest.mark.gpu

NAMES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
ACTS = {"none": b.WFQ_ACT_NONE, "relu": b.WFQ_ACT_RELU, "silu": b.WFQ_ACT_SILU, "gelu": b.WFQ_ACT_GELU}
SHAPES = [10000 * s + 1000 + bn for s in (1, 2, 4, 8) for bn in (64, 128)] + \
         [10000 * s + 2000 + bn for s in (1, 2, 4, 8) for bn in (16, 32, 64)] + [13128, 13256, 14004]


def _rand(shape, dtype, seed, size=1.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=gen, device="cuda") * size).to(dtype)


def _case(rows, C, K, gs, dtype="f16", out=None, act="none", bias=False, residual=False, gated=False, shape=0, codes=False,
          seed=0):
    t, o = NAMES[dtype], NAMES[out or dtype]
    x, w = _rand((rows, C), t, seed + 1), _rand(((2 if gated else 1) * K, C), t, seed + 2, C ** -0.5)
    bv = _rand((w.shape[0],), torch.float32, seed + 3, 0.5) if bias else None
    r = _rand((rows, K), o, seed + 4) if residual else None
    layer = b.Linear(C, K, gs, rows, dtype, out_dtype=out, gated=gated)
    layer.prepare(w)
    layer.set_epilogue(bv, ACTS[act])
    if shape:
        b.wfq_linear_set_debug_option(layer.lin, b.WFQ_DEBUG_GEMM_SHAPE, shape)
    y = layer.forward_codes(b.quantize_rows(x, gs), residual=r) if codes else layer.forward(x, residual=r)
    layer.check_status()
    want, tol = ref.linear(*ref.quantize(x, gs), *ref.quantize(w, gs), gs, bv, act, gated, r, o)
    assert y.dtype is o and y.shape == (rows, K)
    off = (y.double().cpu() - want).abs()
    assert (off <= tol).all(), (float((off / tol).max()), int((off > tol).sum()))
    layer.close()


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("rows,C,K,gs", [(200, 1280, 300, 128), (150, 1216, 290, 64), (40, 1056, 140, 32), (130, 1100, 70, 96),
                                         (33, 1536, 129, 256), (17, 2048, 257, 0), (5, 1120, 40, 160), (300, 1024, 520, 512)])
def test_every_kernel_shape(rows, C, K, gs, shape):
    _case(rows, C, K, gs, out="f32", bias=True, shape=shape)


@pytest.mark.parametrize("shape", [11064, 11128, 13128, 13256, 21128, 41064, 12016, 12032, 12064, 22016, 42032, 82064, 14004])
@pytest.mark.parametrize("act", ["none", "relu", "silu", "gelu"])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_epilogues(dtype, gated, act, shape):
    _case(7 if shape == 14004 else 35, 1024, 75, 128, dtype, act=act, bias=True, residual=True, gated=gated, shape=shape, codes=gated)


@pytest.mark.parametrize("shape", [11064, 11128, 13128, 13256])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_residual_over_many_tiles(dtype, gated, shape):
    """Several tiles per CTA, ragged in both directions, with rows of y and the residual that allow wide accesses."""
    _case(1300, 160, 2056, 64, dtype, act="silu", bias=True, residual=True, gated=gated, shape=shape)


@pytest.mark.parametrize("rows", [1, 2, 3, 4, 5, 8, 9, 16, 17, 31, 64, 65, 127, 128, 129, 500])
@pytest.mark.parametrize("C,K,gs,dtype", [(640, 1280, 64, "f16"), (768, 320, 32, "bf16"), (1009, 77, 128, "f32")])
def test_rows(rows, C, K, gs, dtype):
    _case(rows, C, K, gs, dtype, act="silu", bias=True, residual=True, codes=rows % 2 == 0)


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("rows,C,K,gs", [(1, 1, 1, 32), (1, 33, 1, 32), (2, 31, 3, 0), (130, 32, 2, 32), (7, 100, 9, 64),
                                         (1, 4096, 5, 0), (3, 200, 1001, 96), (129, 127, 129, 128), (1, 20000, 64, 128),
                                         (20, 8200, 40, 1024), (2, 131072, 16, 0), (600, 64, 64, 32)])
def test_odd_sizes(rows, C, K, gs, gated):
    _case(rows, C, K, gs, "bf16", out="f32", gated=gated, act="silu" if gated else "none", bias=True)
    _case(rows, C, K, gs, "f32", out="f16", gated=gated, act="relu", residual=True, codes=True)


@pytest.mark.parametrize("in_t", list(NAMES))
@pytest.mark.parametrize("out_t", list(NAMES))
def test_types(in_t, out_t):
    _case(70, 320, 200, 64, in_t, out_t, act="gelu", residual=True)
    _case(3, 320, 200, 64, in_t, out_t, act="gelu", residual=True)


def _layer(C=640, K=256, gs=64, rows=300, dtype="f16", seed=7, **more):
    layer = b.Linear(C, K, gs, rows, dtype, **more)
    layer.prepare(_rand((layer.K * (2 if layer.gated else 1), C), NAMES[dtype], seed, C ** -0.5))
    return layer


@pytest.mark.parametrize("rows", [1, 6, 40, 300])
@pytest.mark.parametrize("ldx,ldy,ldr,offset", [(640, 256, 256, 0), (648, 264, 272, 0), (641, 257, 259, 1), (700, 300, 256, 3)])
@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_strides_and_alignment(dtype, ldx, ldy, ldr, offset, rows):
    t = NAMES[dtype]
    layer = _layer(dtype=dtype)
    x, r = _rand((rows, 640), t, 1), _rand((rows, 256), t, 2)
    want = layer.forward(x, residual=r)

    def place(v, ld, fill):
        flat = torch.full((rows * ld + offset,), fill, dtype=t, device="cuda")
        view = flat[offset:].as_strided(v.shape, (ld, 1))
        view.copy_(v)
        return flat, view
    _, xv = place(x, ldx, 3.0)
    _, rv = place(r, ldr, 4.0)
    flat, yv = place(torch.zeros_like(want), ldy, 5.0)
    layer.forward(xv, residual=rv, y=yv)
    assert torch.equal(yv, want)
    beside = torch.ones_like(flat, dtype=torch.bool)
    beside[offset:].as_strided(want.shape, (ldy, 1)).fill_(False)
    assert (flat[beside] == 5.0).all()                               # nothing beside the rows is written
    _, yr = place(r, ldr, 6.0)                                       # the residual updated in place
    layer.forward(xv, residual=yr, y=yr)
    assert torch.equal(yr, want)


def test_rows_behind_the_last_stay():
    layer = _layer()
    for rows in (1, 5, 33, 129, 299):
        buf = torch.full((300, 256), 8.0, dtype=torch.float16, device="cuda")
        layer.forward(_rand((rows, 640), torch.float16, rows), y=buf[:rows])
        assert (buf[rows:] == 8.0).all() and not (buf[:rows] == 8.0).all(dim=1).any()
    assert layer.forward(_rand((0, 640), torch.float16, 1)).shape == (0, 256)


def test_rows_without_values_and_not_finite():
    layer = _layer(gs=64)
    layer.set_epilogue(_rand((256,), torch.float32, 3), b.WFQ_ACT_NONE)
    for rows in (4, 40, 200):
        x = _rand((rows, 640), torch.float16, rows)
        clean = layer.forward(x)
        x[0] = 0
        x[1, 100] = float("nan")
        x[2, 5] = float("inf")
        y = layer.forward(x)
        assert torch.equal(y[0], layer._bias.half())
        assert torch.isnan(y[1:3]).all()
        assert torch.equal(y[3:], clean[3:])


@pytest.mark.parametrize("size", [1e-28, 1e-20, 1e20, 1e30, 1e33])
@pytest.mark.parametrize("rows", [2, 200])
def test_scales_far_from_one(rows, size):
    """Rows whose scales are near the ends of the 32-bit range; small weights keep the results inside it."""
    x, w = _rand((rows, 256), torch.float32, 1) * size, _rand((96, 256), torch.float32, 2, 1e-3)
    layer = b.Linear(256, 96, 64, rows, "f32")
    layer.prepare(w)
    want, tol = ref.linear(*ref.quantize(x, 64), *ref.quantize(w, 64), 64)
    off = (layer.forward(x).double().cpu() - want).abs()
    assert (off <= tol + 2.0 ** -126).all()


def test_same_bits_again_and_on_another_stream():
    layer = _layer()
    x = _rand((300, 640), torch.float16, 5)
    for rows in (1, 20, 300):
        want = layer.forward(x[:rows])
        assert torch.equal(layer.forward(x[:rows]), want)
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            got = layer.forward(x[:rows])
        side.synchronize()
        assert torch.equal(got, want)


def test_captured_and_replayed():
    layer, other = _layer(), _layer(C=256, K=640, seed=9)
    for rows in (1, 16, 300):
        x = _rand((rows, 640), torch.float16, 5)
        layer.forward(x)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            y = other.forward(layer.forward(x), residual=x)
        for seed in (6, 7):
            x.copy_(_rand((rows, 640), torch.float16, seed))
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(y, other.forward(layer.forward(x), residual=x))


def test_weights_replaced_between_calls():
    """New weights are what the next call uses, whichever kernel runs and whatever it may fetch early."""
    layer = _layer(C=2048, K=1024, gs=128, rows=130)
    ws = [_rand((1024, 2048), torch.float16, s, 0.02) for s in range(4)]
    for rows in (1, 4, 20, 130):
        q = b.quantize_rows(_rand((rows, 2048), torch.float16, rows), 128)
        want = []
        for w in ws:
            layer.prepare(w)
            torch.cuda.synchronize()
            want.append(layer.forward_codes(q))
            torch.cuda.synchronize()
        for _ in range(5):
            got = []
            for w in ws:
                layer.prepare(w)
                got.append(layer.forward_codes(q))
                layer.prepare(w)
                got.append(layer.forward_codes(q))
            for i in range(4):
                assert torch.equal(got[2 * i], want[i]) and torch.equal(got[2 * i + 1], want[i])


def test_prepared_weights():
    for gated in (False, True):
        K, C, gs = 70, 200, 64
        w = _rand(((2 if gated else 1) * K, C), torch.bfloat16, 3)
        layer = b.Linear(C, K, gs, 1, "bf16", gated=gated)
        layer.prepare(w)
        codes, scales = ref.quantize(w, gs)
        if gated:                                                    # gate and value rows alternate
            order = torch.arange(2 * K).reshape(2, K).T.reshape(-1)
            codes, scales = codes[order], scales[order]
        ptr, n = b.wfq_linear_debug_get(layer.lin, b.WFQ_BUF_WQ)
        got = torch.as_tensor(b._DevicePointer(ptr, (len(codes), 224), "|i1"), device="cuda").cpu()
        assert n == got.numel() and torch.equal(got[:, :C].double(), codes) and not got[:, C:].any()
        ptr, n = b.wfq_linear_debug_get(layer.lin, b.WFQ_BUF_SW)
        got = torch.as_tensor(b._DevicePointer(ptr, (4, 256), "<f4"), device="cuda").cpu()
        assert n == got.numel() * 4 and torch.equal(got[:, :len(codes)].T.double(), scales) and not got[:, len(codes):].any()


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("rows,gs", [(1, 64), (7, 128), (300, 64), (129, 0)])
def test_feed_forward_block(rows, gs, dtype):
    """Norm, gated product on its codes, product back onto the stream: each step against 64 bits from what it was given."""
    C, F, t = 640, 1000, NAMES[dtype]
    x, res = _rand((rows, C), t, 1), _rand((rows, C), t, 2)
    gain = 1 + _rand((C,), torch.float32, 3, 0.1)
    wi, wo = _rand((2 * F, C), t, 4, C ** -0.5), _rand((C, F), t, 5, F ** -0.5)
    up, down = b.Linear(C, F, gs, rows, dtype, gated=True), b.Linear(F, C, gs, rows, dtype)
    up.prepare(wi)
    down.prepare(wo)
    up.set_epilogue(None, b.WFQ_ACT_SILU)
    q, h = b.rms_norm_quantize(x, gain, 1e-6, gs, residual=res)
    inner = up.forward_codes(q)
    y = down.forward(inner, residual=h)
    want_h, codes, scales = ref.rms_norm_quantize(x, res, gain, 1e-6, gs)
    assert torch.equal(h.cpu(), want_h) and torch.equal(q.codes[:, :C].cpu().double(), codes)
    got_scales = q.scales[:, :rows].T.double().cpu()
    assert ((got_scales - scales).abs() <= ref.norm_scale_tolerance(C) * scales).all()
    want, tol = ref.linear(codes, got_scales, *ref.quantize(wi, gs), gs, None, "silu", True, None, t)
    assert ((inner.double().cpu() - want).abs() <= tol).all()
    want, tol = ref.linear(*ref.quantize(inner, gs), *ref.quantize(wo, gs), gs, None, "none", False, h, t)
    assert ((y.double().cpu() - want).abs() <= tol).all()
    up.check_status()
    down.check_status()


@pytest.mark.parametrize("stage", [0, 1])
@pytest.mark.parametrize("shape", [s for s in SHAPES if s != 14004])          # no waits in the dot products
def test_starved_product_ends(shape, stage):
    """A stage that is never loaded: the waits run out, the kernel says so and ends, a new layer works."""
    x = _rand((100, 2048), torch.float16, 1)
    layer = _layer(C=2048, K=200, rows=100)
    want = layer.forward(x)
    b.wfq_linear_set_debug_option(layer.lin, b.WFQ_DEBUG_GEMM_SHAPE, shape)
    b.wfq_linear_set_debug_option(layer.lin, b.WFQ_DEBUG_WAIT_CYCLES, 2_000_000)
    b.wfq_linear_set_debug_option(layer.lin, b.WFQ_DEBUG_SKIP_GEMM_STAGE, stage)
    layer.forward(x)
    torch.cuda.synchronize()
    status, where = b.wfq_linear_check_status(layer.lin, torch.cuda.current_stream().cuda_stream)
    assert status == b.WFQ_ERR_TIMEOUT and where in range(1, 7)
    layer.close()
    layer = _layer(C=2048, K=200, rows=100)
    assert torch.equal(layer.forward(x), want)
    layer.check_status()


@pytest.mark.parametrize("rows", [1, 4, 20, 200])
def test_weights_written_by_a_graph(rows):
    """A graph that prepares the weights, and products behind its replays, inside the graph and outside."""
    layer = _layer(C=1024, K=512, gs=128, rows=rows)
    w = _rand((512, 1024), torch.float16, 20, 0.02)
    q = b.quantize_rows(_rand((rows, 1024), torch.float16, rows), 128)
    layer.prepare(w)
    layer.forward_codes(q)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.prepare(w)
        inside = layer.forward_codes(q)
    for seed in range(21, 27):
        w.copy_(_rand((512, 1024), torch.float16, seed, 0.02))
        graph.replay()
        outside = layer.forward_codes(q)
        torch.cuda.synchronize()
        fresh = _layer(C=1024, K=512, gs=128, rows=rows)
        fresh.prepare(w)
        want = fresh.forward_codes(q)
        assert torch.equal(inside, want) and torch.equal(outside, want)


def test_first_preparation_under_capture_is_refused():
    """It allocates, which would end the capture: the call fails, the capture and the layer go on."""
    x = torch.randn(5, 96, device="cuda")
    w = torch.randn(40, 96, device="cuda")
    layer = b.Linear(96, 40, 32, 8, "f32")
    out = torch.zeros(8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        with pytest.raises(b.WfqError) as err:
            layer.prepare(w)
        out += 1
    assert err.value.status == b.WFQ_ERR_INVALID_ARG
    graph.replay()
    assert out.tolist() == [1.0] * 8
    layer.prepare(w)
    assert torch.isfinite(layer.forward(x)).all()
    layer.check_status()


@pytest.mark.parametrize("shape", [s for s in SHAPES if s // 10000 == 1 and s // 1000 % 10 != 4])
@pytest.mark.parametrize("C,gs", [(32, 0), (64, 0), (64, 256), (64, 32), (96, 0), (128, 64), (160, 96), (224, 32)])
def test_few_channels_over_many_tiles(C, gs, shape):
    """Several tiles per CTA, each of one or two stages: every slot of tensor memory is used."""
    _case(1500, C, 4100, gs, "bf16", shape=shape, codes=True, residual=True)
