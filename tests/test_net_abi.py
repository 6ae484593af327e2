"""CPU checks of the network operators' C ABI: exports, the record's layout, and refusals before anything reaches a GPU."""
import ctypes as C
import os
import re

import numpy as np
import pytest
import torch

import net_oracle as O

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P, BAD_ALIGNED = 4096, 4100  # addresses that are never followed


@pytest.fixture(scope="module")
def net():
    from paper_2012_04201_amd import binding, build, net
    if not os.path.exists(binding.LIB_PATH):
        build.build_lib()
    return net


def test_header_symbols_are_exported(net):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "bbo_net.h")).read(), flags=re.S)
    declared = sorted(set(re.findall(r"\b(bbo_net_[a-z_0-9]+)\s*\(", text)))
    assert sorted(net.EXPORTS) == declared
    for s in declared:
        assert hasattr(net.lib(), s), s


def test_record_layout(net):
    T = net.Tensor
    assert C.sizeof(T) == 72 and T.n.offset == 56 and T.lr.offset == 64 and T.weight_decay.offset == 68


def norm(net, x=P, xs=8, r=0, rs=8, w=P, rows=4, width=8, eps=1e-6, dt=0, s=0, ss=8, y=P, ys=8, rstd=0, q=0, qs=128, sc=0, scs=4):
    return net.lib().bbo_net_rms_norm(x, xs, r, rs, w, rows, width, eps, dt, s, ss, y, ys, rstd, q, qs, sc, scs, 0)


def grad(net, dy=P, s=8, dsum=0, h=P, rstd=P, w=P, rows=4, width=8, dt=0, dx=P, dw=P, ws=P, room=1 << 30):
    return net.lib().bbo_net_rms_norm_grad(dy, s, dsum, s, h, s, rstd, w, rows, width, dt, dx, s, dw, ws, room, 0)


def quant(net, x=P, xs=200, gate=0, gs=200, rows=4, cols=200, dt=0, tile=1, q=P, qs=256, s=P, ss=4, qt=0, qts=128, st=0, sts=4):
    return net.lib().bbo_net_quantize(x, xs, gate, gs, rows, cols, dt, tile, q, qs, s, ss, qt, qts, st, sts, 0)


def mm(net, a=P, a_s=256, sa=P, sas=4, at=1, b=P, b_s=256, sb=P, sbs=4, bt=1, m=4, n=8, k=200, c=P, cs=8, dt=0, acc=0, ws=0, room=0):
    return net.lib().bbo_net_matmul8(a, a_s, sa, sas, at, b, b_s, sb, sbs, bt, m, n, k, c, cs, dt, acc, ws, room, 0)


def adam(net, n=10, count=1, p=P, g=P, m=P, v=P, ms=0, vs=0, copy=0, lr=1e-3, wd=0.0, pd=0, gd=0, moments=0, b1=0.9, b2=0.999, eps=1e-8, step=1, table=True):
    t = (net.Tensor * 1)(net.Tensor(p, g, m, v, ms, vs, copy, n, lr, wd))
    return net.lib().bbo_net_adamw(t if table else None, count, pd, gd, moments, b1, b2, eps, step, 0, 0, 0)


INVALID, UNSUPPORTED, SMALL = 1, 2, 3


@pytest.mark.parametrize("call,kw,code", [
    (norm, dict(rows=-1), INVALID), (norm, dict(width=0), INVALID), (norm, dict(width=40000, xs=40000, ys=40000), UNSUPPORTED),
    (norm, dict(dt=7), INVALID), (norm, dict(eps=-1.0), INVALID), (norm, dict(eps=float("nan")), INVALID), (norm, dict(x=0), INVALID),
    (norm, dict(r=P), INVALID), (norm, dict(s=P), INVALID), (norm, dict(q=P), INVALID), (norm, dict(xs=7), INVALID),
    (norm, dict(r=P, s=P, rs=7), INVALID), (norm, dict(q=P, sc=P, qs=7), INVALID), (norm, dict(ys=7), INVALID),
    (grad, dict(rows=-1), INVALID), (grad, dict(dt=2), INVALID), (grad, dict(dy=0), INVALID), (grad, dict(rstd=0), INVALID),
    (grad, dict(dx=0), INVALID), (grad, dict(s=7), INVALID), (grad, dict(ws=0), INVALID), (grad, dict(ws=BAD_ALIGNED), INVALID),
    (grad, dict(room=16), SMALL),
    (quant, dict(rows=-1), INVALID), (quant, dict(tile=64), INVALID), (quant, dict(dt=5), INVALID), (quant, dict(s=0), INVALID),
    (quant, dict(qt=P), INVALID), (quant, dict(x=0), INVALID), (quant, dict(xs=199), INVALID), (quant, dict(qs=199), INVALID),
    (quant, dict(ss=1), INVALID), (quant, dict(gate=P, gs=1), INVALID), (quant, dict(qt=P, st=P, qts=3), INVALID),
    (quant, dict(rows=1 << 40), UNSUPPORTED),
    (mm, dict(m=-1), INVALID), (mm, dict(at=2), INVALID), (mm, dict(bt=0), INVALID), (mm, dict(dt=9), INVALID), (mm, dict(c=0), INVALID),
    (mm, dict(cs=7), INVALID), (mm, dict(a=0), INVALID), (mm, dict(sb=0), INVALID), (mm, dict(a_s=199), INVALID),
    (mm, dict(sbs=1), INVALID), (mm, dict(ws=BAD_ALIGNED, room=64), INVALID), (mm, dict(m=1 << 40), UNSUPPORTED),
    (adam, dict(count=-1), INVALID), (adam, dict(pd=3), INVALID), (adam, dict(moments=2), INVALID), (adam, dict(b1=1.0), INVALID),
    (adam, dict(b2=-0.1), INVALID), (adam, dict(eps=float("nan")), INVALID), (adam, dict(step=0), INVALID), (adam, dict(table=False), INVALID),
    (adam, dict(n=-1), INVALID), (adam, dict(p=0), INVALID), (adam, dict(v=0), INVALID), (adam, dict(moments=1), INVALID),
    (adam, dict(copy=P, pd=1), INVALID), (adam, dict(lr=float("nan")), INVALID)])
def test_refusals(net, call, kw, code):
    assert call(net, **kw) == code
    assert net.lib().bbo_net_last_error()


def test_nothing_to_do_is_no_error(net):
    assert norm(net, rows=0, x=0, y=0, w=0) == 0
    assert quant(net, rows=0, x=0) == 0 and quant(net, cols=0, x=0) == 0 and quant(net, q=0, s=0) == 0
    assert mm(net, m=0, c=0) == 0 and mm(net, n=0, c=0) == 0
    assert adam(net, count=0, table=False) == 0 and adam(net, n=0, p=0, g=0, m=0, v=0) == 0
    assert net.lib().bbo_net_last_error() == b""
    out = net._SZ(7)
    assert net.lib().bbo_net_matmul8_workspace(4, 4, 4, C.byref(out)) == 0
    assert net.lib().bbo_net_matmul8_workspace(-4, 4, 4, C.byref(out)) == INVALID
    assert net.lib().bbo_net_matmul8_workspace(100, 100, 16000, C.byref(out)) == 0 and out.value >= 2 * 100 * 100 * 4
    for m, n, k in ((4096, 4096, 4096), (20000, 20000, 1 << 30), (1, 4096, 128), (0, 5, 5), (5, 0, 5), (5, 5, 0), (2**31 - 1, 2**31 - 1, 2**31 - 1)):
        assert net.lib().bbo_net_matmul8_workspace(m, n, k, C.byref(out)) == 0 and out.value == 0, (m, n, k)
    for m, n, k in ((700, 10000, 100000), (5000, 5000, 10**6), (32, 2000, 10**6), (128, 128, 10**9)):
        assert net.lib().bbo_net_matmul8_workspace(m, n, k, C.byref(out)) == 0 and out.value < 1 << 28, (m, n, k)
    assert net.lib().bbo_net_rms_norm_grad_workspace(3, 100, C.byref(out)) == 0 and out.value >= 100 * 4


def test_binding_refuses_what_the_library_cannot_see(net):
    x = torch.zeros(4, 8)
    for f in (lambda: net.rms_norm(x), lambda: net.quantize(x), lambda: net.rms_norm_grad(x, x, torch.zeros(4)),
              lambda: net.matmul8(net.Blocks8(x, x, 1), net.Blocks8(x, x, 1)), lambda: net.rms_norm(torch.zeros(8)),
              lambda: net.AdamW([x]).step([x]), lambda: net.AdamW([x], state="4bit"),
              lambda: net.AdamW([x, x.bfloat16()]), lambda: net.matmul8(net.Blocks8(x, x, 3), net.Blocks8(x, x, 1))):
        with pytest.raises(ValueError):
            f()


def test_the_oracle_itself():
    """e4m3 against torch's type, the scales' rule, unbiased random rounding."""
    v = O.e4m3_values()
    assert np.array_equal(v, torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy())
    for top, byte in ((448.0, 127), (449.0, 128), (224.0, 126), (1.0, 119), (0.0, 0), (2.0 ** -140, 0), (3e38, 247)):
        assert int(O.scale_bytes(np.array([top]))[0]) == byte, top
    x = np.random.default_rng(1).standard_normal((5, 300)) * 10
    q, b = O.quantize(x, 1)
    s = 2.0 ** (np.repeat(b.astype(float), 128, 1)[:, :300] - 127)
    assert np.array_equal(q, torch.from_numpy((x / s).astype(np.float32)).to(torch.float8_e4m3fn).double().numpy())
    rm, rv = O.random16(O.key_fold(5, 3), 1 << 16)
    assert abs(rm.mean() / 65536 - 0.5) < 5e-3 and abs(rv.mean() / 65536 - 0.5) < 5e-3
    for t in (1.03, 300.0, 2.0 ** -8.5, 2.0 ** -11):
        mean = O.decode(O.round_random(np.full(1 << 16, t, np.float32), rm, 0)).astype(np.float64).mean()
        gap = max(2.0 ** (np.floor(np.log2(t)) - 3), 2.0 ** -9)
        assert abs(mean - t) < gap * (4 * 0.5 / 256 + 2.0 ** -16), (t, mean)  # four standard errors, and the 16 bits
