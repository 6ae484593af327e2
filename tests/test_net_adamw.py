"""GPU tests of the AdamW step: float32 moments against 64 bits, 8-bit moments bit for bit against float32 arithmetic in numpy."""
import numpy as np
import pytest
import torch

import net_oracle as O

pytestmark = pytest.mark.gpu
B1, B2, EPS, LR, WD = 0.9, 0.999, 1e-8, 3e-3, 0.02


@pytest.fixture(scope="module")
def net():
    from paper_2012_04201_amd import net
    net.lib()
    return net


SIZES = [1, 7, 8, 127, 128, 129, 1000, 2047, 2048, 2049, 10007]


def tensors(sizes, p_dtype, g_dtype, seed=0, packed=False):
    g = torch.Generator().manual_seed(seed)
    flat_p, flat_g = torch.randn(sum(sizes), generator=g), torch.randn(sum(sizes), generator=g) * 1e-2
    p, gr = [], []
    at = 0
    P, G = flat_p.to(p_dtype).cuda(), flat_g.to(g_dtype).cuda()
    for n in sizes:
        p.append(P[at:at + n] if packed else P[at:at + n].clone())
        gr.append(G[at:at + n] if packed else G[at:at + n].clone())
        at += n
    return p, gr


def updated(p, m, v, step, lr, wd):
    """(value, bound of float32's error) of the update in 64 bits."""
    u = (m / (1 - B1 ** step)) / (np.sqrt(v / (1 - B2 ** step)) + EPS)
    want = p - lr * wd * p - lr * u
    # p: one product and one difference; u: m and v as above, eight rounded operations, and factors that are float32
    return want, (np.abs(p) * 4 + np.abs(lr * u) * 64) * O.EPS32


@pytest.mark.parametrize("p_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("g_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("packed", [False, True])
def test_float32_moments(net, p_dtype, g_dtype, packed):
    ps, gs = tensors(SIZES, p_dtype, g_dtype, packed=packed)
    copies = [torch.zeros(n, dtype=torch.bfloat16).cuda() for n in SIZES] if p_dtype == torch.float32 else None
    lrs, wds = [LR * (1 + i) for i in range(len(SIZES))], [WD if i % 2 else 0.0 for i in range(len(SIZES))]
    opt = net.AdamW(ps, lr=lrs, betas=(B1, B2), eps=EPS, weight_decay=wds, copies=copies)
    for step in (1, 2, 3):
        before = [(p.cpu().double().numpy(), m.cpu().double().numpy(), v.cpu().double().numpy()) for p, (m, v) in zip(ps, opt.moments)]
        opt.step(gs)
        for i, (p0, m0, v0) in enumerate(before):
            g = gs[i].cpu().double().numpy()
            m, v = B1 * m0 + (1 - B1) * g, B2 * v0 + (1 - B2) * g * g
            got_m, got_v = (t.cpu().double().numpy() for t in opt.moments[i])
            assert (np.abs(got_m - m) <= (np.abs(B1 * m0) + np.abs((1 - B1) * g)) * 4 * O.EPS32).all()
            assert (np.abs(got_v - v) <= v * 5 * O.EPS32 + 1e-45).all()
            want, bound = updated(p0, m, v, step, lrs[i], wds[i])
            got = ps[i].cpu().double().numpy()
            half = O.EPS16 * (1 + 2 ** -7) * np.abs(want) if p_dtype == torch.bfloat16 else 0
            assert (np.abs(got - want) <= bound + half).all()
            if copies:
                assert torch.equal(copies[i], ps[i].bfloat16())
        gs = [g * -0.5 for g in gs] if not packed else gs


@pytest.mark.parametrize("p_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("g_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("packed", [False, True])
def test_8bit_moments_bit_for_bit(net, p_dtype, g_dtype, packed):
    ps, gs = tensors(SIZES, p_dtype, g_dtype, 1, packed)
    copies = [torch.zeros(n, dtype=torch.bfloat16).cuda() for n in SIZES] if p_dtype == torch.float32 else None
    opt = net.AdamW(ps, lr=LR, betas=(B1, B2), eps=EPS, weight_decay=WD, state="8bit", seed=77, copies=copies)
    host = lambda s: [s.m.cpu().view(torch.uint8).numpy().copy(), s.m_scales.cpu().numpy().copy(), s.v.cpu().view(torch.uint8).numpy().copy(), s.v_scales.cpu().numpy().copy()]
    for step in range(1, 5):
        before = [(p.cpu().double().numpy(), host(s)) for p, s in zip(ps, opt.moments)]
        opt.step(gs)
        for i, (p0, (m8, ms, v8, vs)) in enumerate(before):
            g = gs[i].cpu().float().numpy()
            m, v, *want = O.adam8(g, m8, ms, v8, vs, B1, B2, O.key_fold(O.key_fold(77, step), i))
            for name, a, b in zip(("m", "m_scales", "v", "v_scales"), host(opt.moments[i]), want):
                assert np.array_equal(a, b), (step, i, SIZES[i], name, int((a != b).sum()))
            m, v = m.astype(np.float64), v.astype(np.float64)
            p, bound = updated(p0, m, v, step, LR, WD)
            half = O.EPS16 * (1 + 2 ** -7) * np.abs(p) if p_dtype == torch.bfloat16 else 0
            assert (np.abs(ps[i].cpu().double().numpy() - p) <= bound + half).all()
        # gradients that grow and shrink by far, vanish in places, and turn
        gs = [(g * (-30.0 if step == 1 else 1e-3)).roll(1) for g in gs]
        gs[3][:100] = 0
        if packed:
            gs = [g.clone() for g in gs]


def test_8bit_second_moment_keeps_its_smallest(net):
    """Squares of gradients from 2^-70 to 2^40 in one block: none but zero gets the code of zero, however small beside the largest."""
    g = torch.Generator().manual_seed(5)
    grad = torch.randn(1000, generator=g) * 2.0 ** torch.randint(-35, 20, (1000,), generator=g)
    grad[::50] = 0
    p = torch.zeros(1000).cuda()
    opt = net.AdamW([p], lr=LR, betas=(B1, B2), eps=EPS, weight_decay=WD, state="8bit", seed=3)
    zeros8, zeros = np.zeros(1000, np.uint8), np.zeros(8, np.float32)
    opt.step([grad.cuda()])
    s = opt.moments[0]
    want = O.adam8(grad.numpy(), zeros8, zeros, zeros8, zeros, B1, B2, O.key_fold(O.key_fold(3, 1), 0))[4]
    assert np.array_equal(s.v.view(torch.uint8).cpu().numpy(), want)
    assert np.array_equal(want == 0, grad.numpy() == 0)


def test_8bit_second_moment_decays_exactly(net):
    """Without a gradient the second moment keeps its codes, and its scale falls by beta2 a step."""
    p, g = torch.zeros(512).cuda(), torch.randn(512, generator=torch.Generator().manual_seed(4)).cuda()
    opt = net.AdamW([p], betas=(B1, B2), state="8bit")
    opt.step([g])
    codes, scales = opt.moments[0].v.view(torch.uint8).clone(), opt.moments[0].v_scales.cpu().numpy().copy()
    for _ in range(50):
        opt.step([torch.zeros_like(g)])
        scales = scales * np.float32(B2)
        assert torch.equal(opt.moments[0].v.view(torch.uint8), codes)
        assert np.array_equal(np.frexp(opt.moments[0].v_scales.cpu().numpy())[0], np.frexp(scales)[0])
    assert np.array_equal(opt.moments[0].v_scales.cpu().numpy(), scales)


def test_8bit_moments_follow_a_long_run(net):
    """After a thousand steps with noisy gradients the 8-bit second moments are the float32 ones on the average, as far as
    e4m3's normal numbers reach below the block's largest (2^-6 of its scale): the mean of their ratio is within four of its
    standard errors (each value's share of rounding noise is under 0.35, the gradients' own spread cancels in the
    ratio).  Below that the least code is the floor: moments are larger on the average, so that steps are smaller."""
    n = 4096
    gen = torch.Generator(device="cuda").manual_seed(5)
    size = torch.logspace(-2, 1, n, device="cuda")[torch.randperm(n, generator=gen, device="cuda")]
    a, b = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    oa, ob = net.AdamW([a], lr=1e-3, weight_decay=0.0), net.AdamW([b], lr=1e-3, weight_decay=0.0, state="8bit")
    for _ in range(1000):
        g = torch.randn(n, generator=gen, device="cuda") * size + 0.3 * size
        oa.step([g])
        ob.step([g])
    scale = ob.moments[0].v_scales.repeat_interleave(128)
    v = oa.moments[0][1]
    ratio = (ob.moments[0].v.float() * scale / v).double()
    normal = v >= scale * 2.0 ** -6
    assert int(normal.sum()) > n // 2
    assert abs(float(ratio[normal].mean()) - 1) < 4 * 0.35 / int(normal.sum()) ** 0.5
    assert float(ratio[~normal].mean()) > 1
    assert float((b - a)[normal].norm() / a[normal].norm()) < 0.35 / 2  # steps go by the moment's root


def test_values_that_are_not_finite_stay_where_they_are(net):
    p, g = torch.zeros(300).cuda(), torch.full((300,), 0.5).cuda()
    g[7], g[130] = float("nan"), float("inf")
    for state in ("f32", "8bit"):
        q = p.clone()
        opt = net.AdamW([q], state=state)
        opt.step([g])
        opt.step([torch.ones_like(g)])
        bad = ~torch.isfinite(q.cpu())
        assert bad.nonzero().view(-1).tolist() == [7, 130]


def test_grad_scale_many_tensors_and_empty_ones(net):
    """More tensors than one launch takes, empty ones among them; the gradient's factor is a device value."""
    sizes = [(37 * i) % 301 for i in range(101)]
    ps, gs = tensors(sizes, torch.float32, torch.float32, 6)
    qs = [p.clone() for p in ps]
    for state in ("f32", "8bit"):
        a, b = net.AdamW(ps, state=state, seed=3), net.AdamW(qs, state=state, seed=3)
        a.step(gs, grad_scale=torch.tensor([0.25]).cuda())
        b.step([g * 0.25 for g in gs])
        assert all(torch.equal(p, q) for p, q in zip(ps, qs))
        flat = lambda o: [t.view(torch.uint8) for s in o.moments for t in s]
        assert all(torch.equal(x, y) for x, y in zip(flat(a), flat(b)))


def test_refusals(net):
    p, g = torch.zeros(10).cuda(), torch.zeros(10).cuda()
    opt = net.AdamW([p])
    for bad in ([], [g[:5]], [g.cpu()], [g.half()], [torch.zeros(20).cuda()[::2]]):
        with pytest.raises(ValueError):
            opt.step(bad)
    assert opt.steps == 0
    for kw in (dict(copies=[torch.zeros(10).cuda()]), dict(lr=[1.0, 2.0]), dict(moments=[]), dict(moments=[(p, p[:5])])):
        with pytest.raises(ValueError):
            net.AdamW([p], **kw)
    with pytest.raises(net.BboError):
        net.AdamW([p], betas=(1.0, 0.9)).step([g])


def test_another_stream_and_a_graph(net):
    ps, gs = tensors(SIZES, torch.float32, torch.bfloat16, 7)
    for state in ("f32", "8bit"):
        a, b = net.AdamW([p.clone() for p in ps], state=state), net.AdamW([p.clone() for p in ps], state=state)
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        a.step(gs)
        b.step(gs, stream=side)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(a.params, b.params))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):  # the step's number is the captured one
            b.step(gs)
        for _ in range(3):
            graph.replay()
            torch.cuda.synchronize()
            a.steps = 1
            a.step(gs)
            torch.cuda.synchronize()
            assert all(torch.equal(x, y) for x, y in zip(a.params, b.params))
