"""GPU tests of the wide network that runs the 8-bit operators together."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def refit():
    from paper_2012_04201_amd import net, refit
    net.lib()
    return refit


def reference(model, x, y):
    """Loss and gradients of the same network in 64 bits on the CPU."""
    w = [t.detach().cpu().double().requires_grad_() for t in model.w]
    norms = [t.detach().cpu().double().requires_grad_() for t in model.norms]
    norm = lambda h, s: h * torch.rsqrt((h * h).mean(1, keepdim=True) + 1e-6) * s
    h = x.cpu().double() @ w[0].t()
    for i in range(model.blocks):
        h = h + torch.relu(norm(h, norms[i]) @ w[2 * i + 1].t()) @ w[2 * i + 2].t()
    out = norm(h, norms[-1]) @ w[-1].t()
    loss = torch.nn.functional.cross_entropy(out, y.cpu()) if model.outputs > 1 else (out - y.cpu().double()[:, None]).square().mean() / 2
    return out.detach(), loss.detach(), torch.autograd.grad(loss, w + norms)


@pytest.mark.parametrize("rows,inputs,outputs,width,hidden,blocks", [(200, 30, 10, 256, 384, 2), (333, 64, 1, 200, 130, 1), (1, 5, 3, 128, 128, 2), (150, 17, 4, 129, 1, 0)])
def test_gradients_follow_64_bits(refit, rows, inputs, outputs, width, hidden, blocks):
    g = torch.Generator().manual_seed(rows)
    model = refit.WideNetwork(inputs, outputs, width, hidden, blocks, seed=1)
    x = torch.randn(rows, inputs, generator=g).bfloat16().cuda()
    y = (torch.randint(0, outputs, (rows,), generator=g) if outputs > 1 else torch.randn(rows, generator=g)).cuda()
    loss, grads = model.gradients(x, y)
    want_out, want_loss, want = reference(model, x, y)
    # every operand is rounded to e4m3, 2.6 % of its size at the root mean square: each of the products on the way (up to
    # 2 + 2 * blocks forward and as many back, two operands each) adds that much at random
    share = 0.026 * (2 * 2 * (2 + 2 * blocks)) ** 0.5
    got = model.predict(x).cpu().double()
    assert float((got - want_out).norm() / want_out.norm()) < 2 * share
    assert abs(float(loss) - float(want_loss)) < 2 * share * max(1.0, float(want_loss))
    for i, (a, b) in enumerate(zip(grads, want)):
        assert a.dtype == torch.float32 and a.shape == b.shape
        # twice that, and for a gradient of few rows the loss's derivative moves with the outputs as a whole
        assert float((a.cpu().double() - b).norm() / b.norm().clamp(min=1e-12)) < 4 * share, i


def test_it_learns_and_serves(refit):
    from paper_2012_04201_amd import inputs
    model, r = refit.refit(inputs.make_config(1, B=1), width=256, hidden=512, blocks=2, epochs=12, batch=256, seed=2)
    assert r["loss"][-1] < 0.1 * r["loss"][0] and r["score"] > 0.9
    x = torch.randn(70, 64, generator=torch.Generator().manual_seed(3)).bfloat16().cuda()
    many = model.predict(x).cpu()
    # one row or many: other kernels, sums in another order, whose roundings to 8 bits may fall on the other side
    for i in (0, 33, 69):
        one = model.predict(x[i:i + 1].contiguous()).cpu()
        assert float((one[0] - many[i]).norm() / many[i].norm()) < 0.1
    again, r2 = refit.refit(inputs.make_config(1, B=1), width=256, hidden=512, blocks=2, epochs=2, batch=256, seed=2)
    assert r2["loss"] == r["loss"][:2]  # the same bits from the same seed


@pytest.mark.parametrize("rows", [1, 5, 64])
def test_served_from_a_graph(refit, rows):
    g = torch.Generator().manual_seed(6)
    model = refit.WideNetwork(30, 4, 256, 300, 2, seed=5)
    serve = model.server(rows)
    for i in range(4):
        x = torch.randn(rows, 30, generator=g).bfloat16().cuda()
        got = serve(x).clone()
        torch.cuda.synchronize()
        assert torch.equal(got, model.predict(x))
        torch.cuda.synchronize()
    before = serve(x).clone()
    model.step(torch.randn(100, 30, generator=g).bfloat16().cuda(), torch.randint(0, 4, (100,), generator=g).cuda())
    assert torch.equal(serve(x).clone(), before)  # the weights of its making
    assert torch.equal(model.server(rows)(x).clone(), model.predict(x)) and not torch.equal(model.predict(x), before)


def test_it_fits_values(refit):
    g = np.random.default_rng(4)
    X = g.normal(size=(600, 13)).astype(np.float32)
    cfg = {"X": X, "y": np.tanh(X[:, 0] * X[:, 1]).astype(np.float32), "n_classes": 0, "fold_idx": np.arange(600) % 5}
    _, r = refit.refit(cfg, width=256, hidden=256, blocks=1, epochs=30, batch=100)
    assert r["loss"][-1] < 0.5 * r["loss"][0]


def test_refusals(refit):
    for sizes in ((0, 1, 8, 8), (4, 0, 8, 8), (4, 1, 0, 8), (4, 1, 8, 0)):
        with pytest.raises(ValueError):
            refit.WideNetwork(*sizes)
    with pytest.raises(ValueError):
        refit.WideNetwork(4, 2, blocks=-1)
