"""The network operators' Python side: what it refuses, what it raises for the library, and that it keeps nothing."""
import sys

import pytest
import torch


@pytest.fixture(scope="module")
def net():
    from paper_2012_04201_amd import net
    net.lib()
    return net


def test_what_is_no_tensor_is_refused(net):
    x = torch.zeros(4, 8)
    for f in (lambda: net.rms_norm(x, weight=3), lambda: net.rms_norm(x, residual=[1]), lambda: net.quantize(x, tile="1"),
              lambda: net.matmul8((x, x, 1), (x, None, 1)), lambda: net.rms_norm(torch.zeros(4, 8, 2)), lambda: net.quantize(x.half())):
        with pytest.raises(ValueError):
            f()
    with pytest.raises(TypeError):
        net._ext.rms_norm(x)


def test_no_parameters(net):
    opt = net.AdamW([])
    opt.step([])
    assert opt.steps == 0
    with pytest.raises(ValueError):
        opt.step([torch.zeros(3)])


@pytest.mark.gpu
def test_refusals_on_the_gpu(net):
    x, w = torch.zeros(4, 8).cuda(), torch.ones(8).cuda()
    q = net.quantize(x)[0]
    rstd = torch.ones(4).cuda()
    for f in (lambda: net.rms_norm(x, w[:7]), lambda: net.rms_norm(x, w.bfloat16()), lambda: net.rms_norm(x, w.cpu()),
              lambda: net.rms_norm(x, residual=x.bfloat16()), lambda: net.rms_norm(x, residual=x[:3]), lambda: net.rms_norm(x.t()),
              lambda: net.rms_norm_grad(x, x, rstd[:3]), lambda: net.rms_norm_grad(x, x, rstd, workspace=torch.zeros(1000)),
              lambda: net.rms_norm_grad(x, x, rstd, dsum=x.cpu()), lambda: net.quantize(x, tile=64), lambda: net.quantize(x, gate=x[:, :7]),
              lambda: net.matmul8(q, q, dtype=torch.float16), lambda: net.matmul8(q, q, accumulate=True),
              lambda: net.matmul8(q, q, out=torch.zeros(4, 5).cuda()), lambda: net.matmul8(q, q, out=torch.zeros(4, 4)),
              lambda: net.matmul8(q, q, workspace=torch.zeros(9)), lambda: net.matmul8(q, net.quantize(x[:, :7])[0]),
              lambda: net.matmul8(q, net.Blocks8(q.values, q.scales, 128)), lambda: net.matmul8(q, net.Blocks8(x, q.scales, 1)),
              lambda: net.AdamW([w]).step([w.cpu()]), lambda: net.AdamW([w]).step([w[:7]]), lambda: net.AdamW([w]).step([w, w]),
              lambda: net.AdamW([w]).step([w], grad_scale=torch.ones(2).cuda())):
        with pytest.raises(ValueError):
            f()
    with pytest.raises(net.BboError):  # the library's own refusal
        net.rms_norm(x, eps=-1.0)
    with pytest.raises(net.BboError):
        net.rms_norm_grad(x, x, rstd, workspace=torch.zeros(4, dtype=torch.uint8).cuda())
    opt = net.AdamW([w.clone()], betas=(0.9, 1.0))
    with pytest.raises(net.BboError):
        opt.step([w])
    assert opt.steps == 0


@pytest.mark.gpu
def test_nothing_is_kept(net):
    """Neither objects nor memory after a call, one that fails included; the output given is the one returned."""
    x, w = torch.randn(4, 256).cuda(), torch.ones(256).cuda()
    q, out = net.quantize(x)[0], torch.zeros(4, 4).cuda()
    ps = [torch.zeros(300).cuda()]
    opt, gs = net.AdamW(ps, state="8bit"), [torch.ones(300).cuda()]
    assert net.matmul8(q, q, out=out) is out

    def all_of_them():
        f = net.rms_norm(x, w, residual=x, want_rstd=True, want_8bit=True)
        net.rms_norm_grad(x, f.sum, f.rstd, w, dsum=x)
        net.quantize(x, gate=x, want_cols=True)
        net.matmul8(q, q)
        net.matmul8(q, q, out=out, accumulate=True)
        opt.step(gs)
        with pytest.raises(net.BboError):
            net.rms_norm(x, w, eps=-1.0, want_8bit=True)
    all_of_them()
    things = [x, w, q.values, q.scales, out, ps[0], gs[0], None, True, False]
    counts, bytes_ = [sys.getrefcount(t) for t in things[:7]], torch.cuda.memory_allocated()
    for _ in range(50):
        all_of_them()
    assert [sys.getrefcount(t) for t in things[:7]] == counts and torch.cuda.memory_allocated() == bytes_


@pytest.mark.gpu
def test_parameters_may_move_and_rates_change(net):
    """A step goes to the tensors that the lists hold now, with the rates of now."""
    ps, gs = [torch.zeros(5).cuda(), torch.zeros(7).cuda()], [torch.ones(5).cuda(), torch.ones(7).cuda()]
    opt = net.AdamW(ps, lr=[0.1, 0.2], weight_decay=0.0)
    opt.step(gs)
    assert torch.allclose(ps[0], torch.full_like(ps[0], -0.1)) and torch.allclose(ps[1], torch.full_like(ps[1], -0.2))
    opt.params[0] = moved = ps[0].clone()
    opt.lr[0] = 0.0
    opt.step(tuple(gs))
    assert torch.allclose(moved, torch.full_like(moved, -0.1)) and torch.allclose(ps[1], torch.full_like(ps[1], -0.4))
    opt.params[0] = torch.zeros(6).cuda()
    with pytest.raises(ValueError):
        opt.step(gs)
