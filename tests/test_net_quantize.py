"""GPU tests of the 8-bit blocks against a definition in 64 bits: every code and scale is the same."""
import numpy as np
import pytest
import torch

import net_oracle as O

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def net():
    from paper_2012_04201_amd import net
    net.lib()
    return net


def data(rows, cols, dtype, seed=0):
    g = torch.Generator().manual_seed(1000 * rows + cols + seed)
    x = (torch.randn(rows, cols, generator=g) * (2 * torch.randn(rows, 1, generator=g)).exp()).to(dtype)
    return x, torch.randn(rows, cols, generator=g).to(dtype)


def same(b, x, tile):
    q, s = O.quantize(x, tile)
    assert np.array_equal(b.scales.cpu().contiguous().view(torch.uint8).numpy(), s)
    assert np.array_equal(b.values.cpu().double().numpy(), q, equal_nan=True)


@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 128), (2, 7), (3, 129), (128, 128), (127, 255), (130, 40), (300, 517), (16, 1024), (1, 5000), (777, 3)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("tile", [1, 128])
@pytest.mark.parametrize("gated", [False, True])
def test_codes_and_scales(net, rows, cols, dtype, tile, gated):
    x, gate = data(rows, cols, dtype)
    want = x.double()
    if gated:
        want = torch.where(gate > 0, want, 0.0)
    want = want.numpy()
    gate = gate.cuda() if gated else None
    q, qt = net.quantize(x.cuda(), tile, gate=gate, want_cols=True)
    same(q, want, tile)
    same(qt, want.T, tile)
    a, none = net.quantize(x.cuda(), tile, gate=gate)
    assert none is None
    same(a, want, tile)
    none, b = net.quantize(x.cuda(), tile, gate=gate, want_rows=False, want_cols=True)
    assert none is None
    same(b, want.T, tile)


@pytest.mark.parametrize("tile", [1, 128])
def test_many_tiles(net, tile):
    """As many as give a thread eight rows."""
    x, gate = data(2600, 2499, torch.bfloat16)
    q, qt = net.quantize(x.cuda(), tile, gate=gate.cuda(), want_cols=True)
    want = torch.where(gate > 0, x.double(), 0.0).numpy()
    same(q, want, tile)
    same(qt, want.T, tile)


@pytest.mark.parametrize("tile", [1, 128])
def test_every_size_of_value(net, tile):
    """Ties, subnormal codes, powers of two at the scales' edges, zeros, values far below their block's largest, and what is not finite."""
    rows, cols = 40, 256
    x = torch.zeros(rows, cols)
    k = torch.arange(cols)
    for i, top in enumerate([448.0, 449.0, 448.0 * 2 ** -20, 1.75, 1.7500001, 1.0, 2.0 ** 100, 2.0 ** -118, 2.0 ** -126, 2.0 ** -140, 3.4e38]):
        x[i] = top * (1.0 - (k % 128) / 128.0)
        x[i, 1::2] *= -1
    x[11] = 448 * 2.0 ** (-(k % 128) / 4.0)
    x[12] = (k % 128 + 0.5) * 2.0 ** -10  # halfway between subnormal codes, beside one at the top
    x[12, ::128] = 448
    x[13] = float("nan")
    x[14] = float("inf")
    x[15] = 1.0
    x[15, 3], x[15, 4], x[15, 130] = float("inf"), float("nan"), -float("inf")
    x[16:] = torch.randn(rows - 16, cols, generator=torch.Generator().manual_seed(2)) * 2.0 ** torch.arange(-12, 12)[:, None]
    q, qt = net.quantize(x.cuda(), tile, want_cols=True)
    same(q, x.double().numpy(), tile)
    same(qt, x.double().numpy().T, tile)


def test_relu_keeps_nan(net):
    x = torch.tensor([[1.0, -2.0, float("nan"), 0.0, -0.0, 5.0]])
    got = O.values(net.quantize(x.cuda(), gate=x.cuda())[0])
    assert np.array_equal(got.numpy(), [[1.0, 0.0, float("nan"), 0.0, 0.0, 5.0]], equal_nan=True)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_strides(net, dtype):
    """Input, gate and outputs with gaps between their rows, at odd addresses; nothing is written between the rows."""
    rows, cols = 150, 201
    x, gate = data(rows, cols, dtype, 1)
    wide = lambda t, off, gap: torch.full((rows, cols + gap), 99.0, dtype=dtype).cuda()[:, off:off + cols].copy_(t)
    xs, gs = wide(x, 1, 6), wide(gate, 3, 3)
    want = torch.where(gate > 0, x.double(), 0.0).numpy()
    for tile in (1, 128):
        q, qt = net.quantize(xs, tile, gate=gs, want_cols=True)
        same(q, want, tile)
        same(qt, want.T, tile)
        room = torch.full((rows, 211), 55, dtype=torch.uint8).cuda()
        scales = torch.full((rows, 5), 55, dtype=torch.uint8).cuda()
        room_t = torch.full((cols, 157), 55, dtype=torch.uint8).cuda()
        scales_t = torch.full((cols, 3), 55, dtype=torch.uint8).cuda()
        p = lambda t, off=0: t.data_ptr() + off
        net._check(net.lib().bbo_net_quantize(p(xs), xs.stride(0), p(gs), gs.stride(0), rows, cols, net._DTYPES[dtype], tile, p(room, 3), 211, p(scales, 1), 5,
                                              p(room_t, 5), 157, p(scales_t), 3, torch.cuda.current_stream().cuda_stream))
        torch.cuda.synchronize()
        assert torch.equal(room[:, 3:3 + cols].cpu(), q.values.cpu().view(torch.uint8)) and (room[:, :3] == 55).all() and (room[:, 3 + cols:] == 55).all()
        assert torch.equal(room_t[:, 5:5 + rows].cpu(), qt.values.cpu().view(torch.uint8)) and (room_t[:, :5] == 55).all() and (room_t[:, 5 + rows:] == 55).all()
        n = -(-rows // tile)
        assert torch.equal(scales[:n, 1:3].cpu(), q.scales.cpu().view(torch.uint8)) and (scales[:, 0] == 55).all() and (scales[n:] == 55).all()
        m = -(-cols // tile)
        assert torch.equal(scales_t[:m, :2].cpu(), qt.scales.cpu().view(torch.uint8)) and (scales_t[:, 2] == 55).all() and (scales_t[m:] == 55).all()


def test_no_values(net):
    q, qt = net.quantize(torch.zeros(0, 5).cuda(), want_cols=True)
    assert q.values.shape == (0, 5) and qt.values.shape == (5, 0) and q.scales.shape == (0, 1) and qt.scales.shape == (5, 0)


def test_another_stream_and_a_graph(net):
    x = data(300, 400, torch.bfloat16, 3)[0].cuda()
    step = lambda stream=None: [t.view(torch.uint8) for b in net.quantize(x, gate=x, want_cols=True, stream=stream) for t in (b.values, b.scales)]
    want = [t.clone() for t in step()]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = step(side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for k in range(3):
        x.copy_(x.roll(k, 0))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip([t.clone() for t in out], step()))
        torch.cuda.synchronize()
