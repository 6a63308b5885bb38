"""The gated delta rule's gradients against central differences of its own forward call, one input at a time.

The loss is sum(O dO) + sum(S_out dS) in 64 bits of fp32 outputs.  Each input is moved along its own gradient, so that the slope is that gradient's norm and no
other's part can stand in for it.  Tolerances, before any run: what the outputs' roundings may move a loss by is, output by output, 9e-6 of its size (as the norms of
test_delta_gpu: 4 sqrt(12 128) 2^-24) times its upstream gradient's; two sizes of the step as Richardson takes them, (4 d(h) - d(2 h)) / 3, have 5 / 3 of that over h
at the most.  The steps' truncation is worked out in 64 bits beside it.  Both together have to be
below 5 % of the slope, so that a gradient of zeros, of the other sign, of half the size or without one of its terms cannot pass."""
import numpy as np
import pytest
import torch

from oracle import delta as R
from paper_2406_08128_amd import binding
from test_delta_gpu import F32, f64, gen, inputs

pytestmark = pytest.mark.gpu
NAMES = ("q", "k", "v", "g", "beta", "S")


@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("H,Hk,dk,dv,T,decay", [(2, 1, 64, 64, 70, 2.0), (1, 1, 128, 64, 45, 1.0), (2, 2, 64, 128, 1100, 5.0)])
def test_each_input_along_its_own_gradient(H, Hk, dk, dv, T, decay, name):
    r = gen(91 + T)
    x = list(inputs(r, T, H, Hk, dk, dv, F32, decay=decay))
    dO, S, dS = x.pop(), 0.3 * r(1, H, dk, dv), 0.3 * r(1, H, dk, dv)
    leaves = dict(zip(NAMES, x + [S]))
    grads = dict(zip(NAMES, binding.chela_gated_delta_bwd(*x, dO, S_in=S, dS_out=dS, want_dS_in=True)))
    grad, leaf = grads[name].double(), leaves[name]
    # (as long as the tensor itself: a step of 1 would move it by its own norm)
    way = grad / grad.norm() * leaf.double().norm()
    share = H // Hk

    def outputs(h):
        y = dict(leaves)
        y[name] = (leaf.double() + h * way).float()
        S_out = torch.empty_like(S)
        O = binding.chela_gated_delta_fwd(*(y[n] for n in NAMES[:5]), S_in=y["S"], S_out=S_out)[0]
        return y, O, S_out

    def loss(h):
        _, O, S_out = outputs(h)
        return float((O.double() * dO.double()).sum() + (S_out.double() * dS.double()).sum())

    def exact(h):
        y = {n: f64(t) for n, t in leaves.items()}
        y[name] = y[name] + h * f64(way)
        at = 0.0
        for i in range(H):
            O, s = R.delta_fwd(y["q"][:, i // share], y["k"][:, i // share], y["v"][:, i], y["g"][:, i], y["beta"][:, i], 1.0, y["S"][0, i])
            at += (O * f64(dO)[:, i]).sum() + (s * f64(dS)[0, i]).sum()
        return at

    def richardson(f, h):
        d1, d2 = ((f(k * h) - f(-k * h)) / (2 * k * h) for k in (1, 2))
        return (4 * d1 - d2) / 3

    h = 0.1
    slope = float((grad * way).sum())
    _, O, S_out = outputs(0.0)
    size = float(O.double().norm() * dO.double().norm() + S_out.double().norm() * dS.double().norm())
    noise = 4 * np.sqrt(12 * 128) * 2.0 ** -24 * size / h * 5 / 3
    # (the inputs moved are rounded to fp32 too: 2^-24 of them, along any direction)
    noise += 2.0 ** -24 * float(leaf.double().norm()) * float(grad.norm()) / h * 5 / 3
    truth = (_definition(x, dO, S, dS, name, share) * f64(way)).sum()
    truncation = abs(richardson(exact, h) - truth)
    assert noise + truncation <= 0.05 * abs(slope), (noise, truncation, slope)
    got = richardson(loss, h)
    assert abs(got - slope) <= noise + truncation, (got, slope, noise, truncation)


def _definition(x, dO, S, dS, name, share):
    q, k, v, g, beta = (f64(t) for t in x)
    out = {"q": np.zeros_like(q), "k": np.zeros_like(k), "v": np.zeros_like(v), "g": np.zeros_like(g), "beta": np.zeros_like(beta), "S": np.zeros_like(f64(S))}
    for i in range(v.shape[1]):
        d = R.delta_bwd(q[:, i // share], k[:, i // share], v[:, i], g[:, i], beta[:, i], f64(dO)[:, i], 1.0, f64(S)[0, i], f64(dS)[0, i])
        out["q"][:, i // share] += d["dQ"]
        out["k"][:, i // share] += d["dK"]
        out["v"][:, i], out["g"][:, i], out["beta"][:, i], out["S"][0, i] = d["dV"], d["dg"], d["dbeta"], d["dS_in"]
    return out[name]
