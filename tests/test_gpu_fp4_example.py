"""The FFN sublayer of examples/fp4_ffn.py: one training step against the same
step in float64 with the plain definitions (quantisation, masks and dropout exact;
activations and activation gradients rounded to bf16 where the example holds
them so), and a short training run."""
import importlib.util
import os

import numpy as np
import pytest

import fp4_plain as P

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    spec = importlib.util.spec_from_file_location("fp4_ffn", os.path.join(ROOT, "examples", "fp4_ffn.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def host(t):
    torch.cuda.synchronize()
    return t.float().cpu().numpy()


@pytest.mark.parametrize("fmt", ["mx", "nv"])
def test_step_matches_the_plain_definitions(fmt):
    """Each stage is checked from the inputs the GPU had for it, so the tolerances are those of one stage: a bf16
    rounding (2^-8) of each output and of the bf16 operand of a gradient, fp32 sums beside it."""
    ex = _example()
    M, d, F, p = 70, 96, 200, 0.2
    layer = ex.FfnSublayer(d, F, M, fmt, p, seed=3)
    layer.step = 5
    gen = torch.Generator(device="cuda").manual_seed(9)
    x = torch.randn((M, d), generator=gen, device="cuda").to(torch.bfloat16)
    r = torch.randn((M, d), generator=gen, device="cuda")
    g = torch.randn((M, d), generator=gen, device="cuda")
    layer.gamma = 0.75
    out = host(layer.forward(x, r)).astype(np.float64)
    gx, gr = (host(t).astype(np.float64) for t in layer.backward(g))
    G = {k: ex.G_X if k == "x" else ex.G_W for k in "xw"} if fmt == "nv" else {"x": 1.0, "w": 1.0}
    q = lambda a, k: P.quantize(a, fmt, G[k])[2:]
    near = lambda a, b, rel, mag: np.all(np.abs(a - b) <= rel * np.abs(b) + 1e-5 * mag)

    def linear(lin, xin):
        xv, _ = q(host(xin), "x")
        wv, _ = q(host(lin.w), "w")
        return xv.astype(np.float64) @ wv.T.astype(np.float64) + host(lin.b)

    y1 = linear(layer.w1, x)
    assert near(host(layer.w1.y), y1, 2.0 ** -8, np.abs(y1).max())
    k1, s = P.keep(M, F, p, 3, 10)
    u = host(layer.w1.y)
    assert np.array_equal(host(layer.h), torch.from_numpy(np.where(k1, np.maximum(u, 0) * np.float32(s), 0)).to(torch.bfloat16).float().numpy())
    y2 = linear(layer.w2, layer.h)
    assert near(host(layer.w2.y), y2, 2.0 ** -8, np.abs(y2).max())
    k2, s = P.keep(M, d, p, 3, 11)
    assert np.array_equal(out, (np.float32(0.75) * host(r) + np.where(k2, host(layer.w2.y) * np.float32(s), np.float32(0))).astype(np.float64))

    # backward
    gh = host(g)
    assert np.array_equal(gr, np.float32(0.75) * gh)
    assert np.array_equal(host(layer.gv), torch.from_numpy(np.where(k2, gh * np.float32(s), 0).astype(np.float32)).to(torch.bfloat16).float().numpy())
    t = (gh.astype(np.float64) * host(r)).sum()
    assert abs(float(layer.ggamma) - t) <= 2.0 ** -24 * 1026 * np.abs(gh * host(r)).sum()
    for lin, G16, xin in ((layer.w2, host(layer.gv), layer.h), (layer.w1, host(layer.gu), x)):
        (xv, xi), (wv, wi) = q(host(xin), "x"), q(host(lin.w), "w")
        G64 = G16.astype(np.float64)
        want = np.where(xi, G64 @ wv, 0)
        assert near(host(lin.gx), want, 2.0 ** -8, np.abs(want).max())
        want = np.where(wi, G64.T @ xv, 0)
        assert near(host(lin.gw), want, 2.0 ** -20, np.abs(want).max())
        assert near(host(lin.gb), G64.sum(0), 2.0 ** -20, np.abs(G64).sum(0).max())
    live = k1 & (u > 0)
    gu = torch.from_numpy(np.where(live, host(layer.w2.gx) * np.float32(P.keep(1, 1, p, 0, 0)[1]), 0).astype(np.float32)).to(torch.bfloat16).float().numpy()
    assert np.array_equal(host(layer.gu), gu)
    assert np.array_equal(gx, host(layer.w1.gx).astype(np.float64))


@pytest.mark.parametrize("fmt", ["mx", "nv"])
def test_training_and_serving(fmt):
    ex = _example()
    losses, layer, x, r, target = ex.train(fmt, steps=40)
    assert losses[-1] < 0.5 * losses[0]
    layer.w1.pack(), layer.w2.pack()
    # one token and the whole batch take different kernels; both give the sublayer without dropout
    layer.p = 0.0
    whole = host(layer.forward(x, r))
    one = host(layer.serve(x[:1], r[:1]))
    assert np.abs(one - whole[:1]).max() <= 2.0 ** -6 * np.abs(whole[:1]).max() + 0.05
