"""The linear layer on several streams: weights prepared on one and used on others, layers side by side."""
import pytest
import torch

from paper_2412_19867_b200 import binding as b

pytestmark = pytest.mark.gpu


def _rand(shape, seed, size=1.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=gen, device="cuda") * size).half()


@pytest.mark.parametrize("rows", [1, 4, 20, 130])
def test_product_behind_the_preparation_though_another_stream_had_one_in_between(rows):
    """Prepared on A, used on B, then on A with nothing between the preparation and this product on A."""
    C, K = 4096, 2048
    layer = b.Linear(C, K, 128, rows, "f16")
    ws = [_rand((K, C), s, 0.02) for s in range(3)]
    q = b.quantize_rows(_rand((rows, C), rows), 128)
    want = []
    for w in ws:
        layer.prepare(w)
        torch.cuda.synchronize()
        want.append(layer.forward_codes(q))
        torch.cuda.synchronize()
    side = [torch.cuda.Stream(), torch.cuda.Stream()]
    outs = [torch.empty((rows, K), dtype=torch.float16, device="cuda") for _ in range(2)]
    torch.cuda.synchronize()
    for i in range(30):
        w, expected = ws[i % 3], want[i % 3]
        with torch.cuda.stream(side[0]):
            layer.prepare(w)
            done = torch.cuda.Event()
            done.record()
        side[1].wait_event(done)
        with torch.cuda.stream(side[1]):
            layer.forward_codes(q, y=outs[1])
        with torch.cuda.stream(side[0]):
            layer.forward_codes(q, y=outs[0])
        side[0].wait_stream(side[1])                     # new weights behind the products that use the old ones
        torch.cuda.synchronize()
        assert torch.equal(outs[0], expected) and torch.equal(outs[1], expected)
    layer.check_status()


@pytest.mark.parametrize("rows", [1, 6, 40, 300])
def test_codes_on_two_streams_at_once(rows):
    C, K = 2048, 1024
    layer = b.Linear(C, K, 128, rows, "f16")
    layer.prepare(_rand((K, C), 1, 0.02))
    qs = [b.quantize_rows(_rand((rows, C), 10 + i), 128) for i in range(2)]
    want = [layer.forward_codes(q) for q in qs]
    streams, outs = [torch.cuda.Stream(), torch.cuda.Stream()], [[], []]
    torch.cuda.synchronize()
    for _ in range(20):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                outs[i].append(layer.forward_codes(qs[i]))
    torch.cuda.synchronize()
    assert all(torch.equal(y, want[i]) for i in range(2) for y in outs[i])
    layer.check_status()


@pytest.mark.parametrize("rows", [(1, 1), (3, 300), (40, 40), (20, 2000), (700, 900)])
def test_two_layers_on_two_streams_at_once(rows):
    """Each with its own workspace, of kernels that hold tensor memory and of others, pairs of CTAs and clusters among them."""
    layers, xs, res = [], [], []
    for i, (C, K, gs) in enumerate([(2048, 1536, 128), (1152, 4096, 64)]):
        layers.append(b.Linear(C, K, gs, rows[i], "f16"))
        layers[i].prepare(_rand((K, C), i, 0.02))
        xs.append(_rand((rows[i], C), 10 + i))
        res.append(_rand((rows[i], K), 20 + i))
    want = [layers[i].forward(xs[i], residual=res[i]) for i in range(2)]
    streams, outs = [torch.cuda.Stream(), torch.cuda.Stream()], [[], []]
    torch.cuda.synchronize()
    for _ in range(20):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                outs[i].append(layers[i].forward(xs[i], residual=res[i]))
    torch.cuda.synchronize()
    assert all(torch.equal(y, want[i]) for i in range(2) for y in outs[i])
    for layer in layers:
        layer.check_status()
