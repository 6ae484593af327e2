"""GPU tests of the 8-bit product against 64 bits."""
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


def matrix(net, rows, cols, tile, seed, pad=True, scales=(100, 140)):
    """Random codes and scales, with NaN where nothing is to be read."""
    g = torch.Generator().manual_seed(seed)
    kb, sr = -(-cols // 128), -(-rows // tile)
    if pad:
        b = net.Blocks8(torch.full((rows, kb * 128), 0x7f, dtype=torch.uint8).cuda().view(torch.float8_e4m3fn)[:, :cols],
                        torch.full((sr, -(-kb // 4) * 4), 255, dtype=torch.uint8).cuda().view(torch.float8_e8m0fnu)[:, :kb], tile)
    else:  # dense rows, at odd addresses for odd lengths
        b = net.Blocks8(torch.empty(rows, cols, dtype=torch.uint8).cuda().view(torch.float8_e4m3fn),
                        torch.empty(sr, kb, dtype=torch.uint8).cuda().view(torch.float8_e8m0fnu), tile)
    codes = torch.randint(0, 127, (rows, cols), generator=g) | (torch.randint(0, 2, (rows, cols), generator=g) << 7)
    b.values.view(torch.uint8).copy_(codes.to(torch.uint8))
    b.scales.view(torch.uint8).copy_(torch.randint(*scales, tuple(b.scales.shape), generator=g).to(torch.uint8))
    return b


def check(got, a, b, c0=None):
    A, B = O.values(a), O.values(b)
    want, size = A @ B.t(), A.abs() @ B.abs().t()
    if c0 is not None:
        want, size = want + c0.cpu().double(), size + c0.cpu().double().abs()
    half = O.EPS16 if got.dtype == torch.bfloat16 else O.EPS32
    # any order of k float32 additions: (k + 8) half-ulps of the magnitudes' sum; one more rounding.  For bfloat16 each of
    # eight neighbouring products may lose what it has below 2^-13 of the largest of them: seven times that.
    bound = size * ((A.shape[1] + 8) * O.EPS32 + (7 * 2.0 ** -13 if got.dtype == torch.bfloat16 else 0)) + want.abs() * half * (1 + 2 ** -7)
    assert got.shape == want.shape
    bad = (got.cpu().double() - want).abs() > bound
    assert not bad.any(), (int(bad.sum()), float(((got.cpu().double() - want).abs() / bound.clamp(min=1e-300)).max()))


SHAPES = [(1, 1, 1), (1, 16, 128), (1, 1000, 513), (2, 17, 100), (16, 33, 640), (17, 129, 130), (31, 40, 64), (33, 50, 1), (64, 64, 127), (65, 64, 128),
          (100, 70, 129), (128, 256, 256), (130, 300, 569), (257, 255, 384), (300, 513, 1000), (1, 300, 5000), (63, 10, 2049)]


@pytest.mark.parametrize("m,n,k", SHAPES)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("tiles", [(1, 1), (1, 128), (128, 1)])
def test_product(net, m, n, k, dtype, tiles):
    a, b = matrix(net, m, k, tiles[0], 1), matrix(net, n, k, tiles[1], 2)
    check(net.matmul8(a, b, dtype=dtype), a, b)
    c0 = (torch.randn(m, n, generator=torch.Generator().manual_seed(3)) * 10).to(dtype).cuda()
    check(net.matmul8(a, b, out=c0.clone(), accumulate=True), a, b, c0)


@pytest.mark.parametrize("m,n,k", [(1, 50, 301), (20, 70, 129), (150, 90, 333), (260, 130, 257)])
def test_rows_at_any_address(net, m, n, k):
    a, b = matrix(net, m, k, 1, 4, pad=False), matrix(net, n, k, 1, 5, pad=False)
    check(net.matmul8(a, b, dtype=torch.float32), a, b)
    wide = torch.full((m, n + 7), 3.0).cuda()
    net.matmul8(a, b, out=wide[:, 3:3 + n])
    check(wide[:, 3:3 + n], a, b)
    assert (wide[:, :3] == 3).all() and (wide[:, 3 + n:] == 3).all()
    wide = torch.full((m, n + 7), 3.0, dtype=torch.bfloat16).cuda()
    net.matmul8(a, b, out=wide[:, 1:1 + n])
    check(wide[:, 1:1 + n], a, b)
    assert (wide[:, :1] == 3).all() and (wide[:, 1 + n:] == 3).all()


@pytest.mark.parametrize("m,n,k", [(3300, 4000, 300), (2500, 2300, 200), (1000, 3100, 1024)])
def test_many_tiles(net, m, n, k):
    """Larger tiles than the small shapes get, ragged at every edge."""
    a, b = matrix(net, m, k, 1, 6), matrix(net, n, k, 128, 7)
    check(net.matmul8(a, b, dtype=torch.float32), a, b)
    check(net.matmul8(a, b), a, b)
    a, b = matrix(net, m, k, 1, 6, pad=False), matrix(net, n, k, 1, 7, pad=False)
    check(net.matmul8(a, b, dtype=torch.float32), a, b)


@pytest.mark.parametrize("m,n,k", [(3300, 2001, 300), (1000, 3100, 1024), (700, 900, 333), (64, 128, 1), (128, 256, 130), (4352, 4096, 600)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_added_to_inside_and_at_the_edges(net, m, n, k, dtype):
    """Tiles that are inside are added to as a whole, those at an edge value by value; rows of c at any address, and what is beside c untouched."""
    a, b = matrix(net, m, k, 1, 29), matrix(net, n, k, 128, 30)
    wide = (torch.randn(m, n + 3, generator=torch.Generator().manual_seed(31)) * 10).to(dtype).cuda()
    c0, sides = wide[:, 1:1 + n].clone(), (wide[:, :1].clone(), wide[:, 1 + n:].clone())
    net.matmul8(a, b, out=wide[:, 1:1 + n], accumulate=True)
    check(wide[:, 1:1 + n], a, b, c0)
    assert torch.equal(wide[:, :1], sides[0]) and torch.equal(wide[:, 1 + n:], sides[1])


@pytest.mark.parametrize("m,n,k", [(3300, 4000, 385), (3333, 3845, 512), (3400, 3840, 640), (3585, 3601, 900), (3300, 4000, 1024), (6200, 1900, 1151), (4500, 4000, 641),
                                   (4110, 4097, 512), (17000, 1000, 1000)])
def test_many_large_tiles(net, m, n, k):
    """Largest tiles, ragged at every edge; odd and even numbers of blocks, whole and with a part at the end."""
    a, b = matrix(net, m, k, 1, 18), matrix(net, n, k, 128 if k & 1 else 1, 19)
    got = net.matmul8(a, b)
    check(got, a, b)
    c0 = (torch.randn(m, n, generator=torch.Generator().manual_seed(3)) * 10).bfloat16().cuda()
    check(net.matmul8(a, b, out=c0.clone(), accumulate=True), a, b, c0)
    assert all(torch.equal(got, net.matmul8(a, b)) for _ in range(3))


@pytest.mark.parametrize("m", [1, 40, 200])
def test_scales_from_one_end_to_the_other(net, m):
    """Scales down to 2^-127 and up to 2^100, zeros under the largest, and NaN as value and as scale."""
    n, k = 96, 512
    a, b = matrix(net, m, k, 1, 8, scales=(0, 30)), matrix(net, n, k, 1, 9, scales=(210, 227))
    check(net.matmul8(a, b, dtype=torch.float32), a, b)
    a, b = matrix(net, m, k, 1, 10), matrix(net, n, k, 1, 11)
    a.values.view(torch.uint8)[0, 200] = 0x7f
    b.scales.view(torch.uint8)[5, 3] = 255
    got = net.matmul8(a, b, dtype=torch.float32).cpu()
    nan = torch.zeros(m, n, dtype=torch.bool)
    nan[0], nan[:, 5] = True, True
    assert torch.equal(got.isnan(), nan)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("m", [1, 40, 200])
def test_zeros_under_the_largest_scales(net, m, dtype):
    """Blocks of zeros add nothing, whatever their scales; scales far apart from each other meet in a product that is in range."""
    n, k = 96, 640
    a, b = matrix(net, m, k, 1, 32), matrix(net, n, k, 1, 33)
    for block, ea, eb in ((0, 254, 254), (2, 0, 254), (3, 250, 3), (4, 254, 0)):
        a.scales.view(torch.uint8)[:, block], b.scales.view(torch.uint8)[:, block] = ea, eb
    a.values.view(torch.uint8)[:, :128] = 0
    check(net.matmul8(a, b, dtype=dtype), a, b)
    b.values.view(torch.uint8)[:, :128] = 0
    check(net.matmul8(a, b, dtype=dtype), a, b)


def test_nothing_contracted(net):
    a, b = net.empty_blocks8(5, 0), net.empty_blocks8(70, 0)
    assert (net.matmul8(a, b) == 0).all()
    c = torch.ones(5, 70).cuda()
    assert (net.matmul8(a, b, out=c, accumulate=True) == 1).all()
    a, b = net.empty_blocks8(300, 0), net.empty_blocks8(70, 0)
    assert (net.matmul8(a, b) == 0).all()
    assert net.matmul8(net.empty_blocks8(0, 50), net.empty_blocks8(3, 50)).shape == (0, 3)


def test_a_layers_gradients(net):
    """y = x w^T in 8 bits: dx and dw are the products of the 8-bit gradient, which differences of y agree with."""
    g = torch.Generator().manual_seed(12)
    m, n, k = 210, 140, 330
    x, w, dy = torch.randn(m, k, generator=g), torch.randn(n, k, generator=g) * k ** -0.5, torch.randn(m, n, generator=g) * 1e-3
    x8, x8t = net.quantize(x.cuda(), want_cols=True)
    w8, w8t = net.quantize(w.cuda(), tile=128, want_cols=True)
    d8, d8t = net.quantize(dy.cuda(), want_cols=True)
    y, dx, dw = net.matmul8(x8, w8, torch.float32), net.matmul8(d8, w8t, torch.float32), net.matmul8(d8t, x8t, torch.float32)
    check(y, x8, w8)
    check(dx, d8, w8t)
    check(dw, d8t, x8t)
    X, W, D = x.double(), O.values(w8), O.values(d8)
    v = torch.randn(m, k, generator=g, dtype=torch.float64)
    slope = float((D * ((X + v) @ W.t() - X @ W.t())).sum())  # y is linear in x and in w
    dot = dx.cpu().double() * v
    assert abs(slope - float(dot.sum())) <= 1e-5 * float(dot.abs().sum())
    Dt, Xt = O.values(d8t), O.values(x8t)
    u = torch.randn(n, k, generator=g, dtype=torch.float64)
    slope = float((Dt.t() * (Xt.t() @ u.t())).sum())
    dot = dw.cpu().double() * u
    assert abs(slope - float(dot.sum())) <= 1e-5 * float(dot.abs().sum())


def test_accuracy_on_normal_data(net):
    """Relative to the result: float32's rounding of a sum of 1000, and 3e-5 beside the bfloat16 output's rounding of 2^-8 / sqrt(12) to sqrt(3)."""
    g = torch.Generator().manual_seed(17)
    for m in (4, 200):
        a, b = (net.quantize(torch.randn(n, 1000, generator=g).cuda())[0] for n in (m, 300))
        want = O.values(a) @ O.values(b).t()
        assert float((net.matmul8(a, b, dtype=torch.float32).cpu().double() - want).norm() / want.norm()) < 1e-6
        got = net.matmul8(a, b).cpu()
        away = (got.double() - want).abs() > (want.bfloat16().double() - want).abs() + 1e-3 * want.abs()
        assert float(away.double().mean()) < 0.02  # rounded the other way than the exact result would be


@pytest.mark.parametrize("m,n,k", [(1, 100, 16000), (20, 33, 9001), (33, 50, 3000), (100, 100, 16000), (130, 127, 5000), (250, 130, 20001), (2100, 600, 9000)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_the_contracted_index_in_parts(net, m, n, k, dtype):
    """Few tiles and long rows: with the workspace that the product asks for, with some of it and with none."""
    import ctypes as C
    a, b = matrix(net, m, k, 1, 20), matrix(net, n, k, 128, 21)
    need = C.c_size_t()
    assert net.lib().bbo_net_matmul8_workspace(m, n, k, C.byref(need)) == 0 and need.value % (4 * m) == 0 and need.value > 4 * m * n
    c0 = (torch.randn(m, n, generator=torch.Generator().manual_seed(22)) * 10).to(dtype).cuda()
    for size in (need.value, need.value - 1, need.value // 2, 2 * m * (n + 3) * 4, 100, 0):
        ws = torch.full((size + 64,), 255, dtype=torch.uint8).cuda()
        got = net.matmul8(a, b, dtype=dtype, workspace=ws[:size])
        check(got, a, b)
        check(net.matmul8(a, b, out=c0.clone(), accumulate=True, workspace=ws[:size]), a, b, c0)
        assert (ws[size:] == 255).all()
        assert torch.equal(got, net.matmul8(a, b, dtype=dtype, workspace=ws[:size]))
    wide = torch.full((m, n + 5), 3.0, dtype=dtype).cuda()
    net.matmul8(a, b, out=wide[:, 1:1 + n])
    check(wide[:, 1:1 + n], a, b)
    assert (wide[:, :1] == 3).all() and (wide[:, 1 + n:] == 3).all()


def test_parts_in_a_graph(net):
    a, b = matrix(net, 70, 9000, 1, 23), matrix(net, 90, 9000, 1, 24)
    graph = torch.cuda.CUDAGraph()
    net.matmul8(a, b)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        out = net.matmul8(a, b)
    for i in range(3):
        b.scales.view(torch.uint8).copy_(b.scales.view(torch.uint8).roll(1, 0))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out.clone(), net.matmul8(a, b))
        torch.cuda.synchronize()


def test_rows_of_scales_far_apart(net):
    """Rows of scales at strides that do not fit the kernels' 32-bit offsets."""
    m, n, k = 70, 2, 520
    a, b = matrix(net, m, k, 1, 25), matrix(net, n, k, 1, 26)
    far = torch.zeros((n - 1) * (1 << 32) + 8, dtype=torch.uint8, device="cuda").as_strided((n, 5), (1 << 32, 1))
    far.copy_(b.scales.view(torch.uint8))
    check(net.matmul8(a, net.Blocks8(b.values, far.view(torch.float8_e8m0fnu), 1), dtype=torch.float32), a, b)
    check(net.matmul8(net.Blocks8(b.values, far.view(torch.float8_e8m0fnu), 1), a, dtype=torch.float32), b, a)


@pytest.mark.parametrize("m", [3, 70])
def test_rows_far_apart(net, m):
    """Rows of values and of the output at strides past 2^32 bytes."""
    n, k = 2, 520
    a, b = matrix(net, m, k, 1, 27), matrix(net, n, k, 1, 28)
    far = torch.zeros((1 << 32) + 1024, dtype=torch.uint8, device="cuda").as_strided((n, k), ((1 << 32) + 16, 1))
    far.copy_(b.values.view(torch.uint8))
    b = net.Blocks8(far.view(torch.float8_e4m3fn), b.scales, 1)
    check(net.matmul8(a, b, dtype=torch.float32), a, b)
    out = torch.zeros((1 << 31) + 4096, dtype=torch.bfloat16, device="cuda").as_strided((n, m), ((1 << 31) + 1, 1))
    check(net.matmul8(b, a, out=out), b, a)
    check(net.matmul8(b, a, out=out.zero_(), accumulate=True), b, a)


def test_the_same_call_gives_the_same_bits(net):
    for m, n, k in ((3, 200, 4000), (100, 100, 4000), (500, 600, 700)):
        a, b = matrix(net, m, k, 1, 13), matrix(net, n, k, 1, 14)
        first = net.matmul8(a, b, dtype=torch.float32)
        assert all(torch.equal(first, net.matmul8(a, b, dtype=torch.float32)) for _ in range(3))


def test_another_stream_and_a_graph(net):
    for m, n, k in ((2, 300, 3000), (200, 300, 600)):
        a, b = matrix(net, m, k, 1, 15), matrix(net, n, k, 1, 16)
        want = net.matmul8(a, b)
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        got = net.matmul8(a, b, stream=side)
        side.synchronize()
        assert torch.equal(got, want)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = net.matmul8(a, b)
        for i in range(3):
            b.scales.view(torch.uint8).copy_(b.scales.view(torch.uint8).roll(i, 0))
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out.clone(), net.matmul8(a, b))
            torch.cuda.synchronize()
