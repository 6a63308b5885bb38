"""The gradient of the log decays on the GPU, token by token (oracle.delta.delta_bounds, dg_divided: followed through the formulas, every term with the
factor e^g_t, on top of it half a step of the output's type): nothing where nothing is let through, and all its digits where little is."""
import numpy as np
import pytest
import torch

from oracle import delta as R
from paper_2406_08128_amd import binding
from test_delta_gpu import BF, DTYPES, compare, cu_of, f64, gen, inputs, offsets

pytestmark = pytest.mark.gpu


def check_dg(dg, x, S, dS, lens, dtype):
    q, k, v, g, beta, dO = (f64(t) for t in x)
    share, o = v.shape[1] // k.shape[1], offsets(lens)
    chunk, once, twice = (64, 2.0 ** -8, 2.0 ** -16) if dtype == BF else (32, 0.0, 0.0)
    for i, (a, b) in enumerate(zip(o, o[1:])):
        for h in range(v.shape[1] if b > a else 0):
            args = (q[a:b, h // share], k[a:b, h // share], v[a:b, h], np.maximum(g[a:b, h], -1e4), beta[a:b, h], dO[a:b, h])
            st, ds = None if S is None else f64(S[i, h]), None if dS is None else f64(dS[i, h])
            ref = R.delta_bwd(*args[:5], args[5], 1.0, st, ds)["dg"]
            compare((i, h), dg[a:b, h], ref, R.delta_bounds(*args, chunk, once, twice, 1.0, st, ds)["dg_divided"])


CASES = [  # H, Hk, dk, dv, lengths, states
    (2, 2, 64, 64, [150], True),
    (2, 1, 64, 128, [64, 0, 33, 1], True),
    (1, 1, 128, 64, [129], False),
    (2, 1, 128, 128, [97, 31], True),
    (1, 1, 64, 64, [1400], False),                 # (runs of several chunks)
    (1, 1, 128, 128, [600, 577], False),
]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("decay", [-2.0, 0.0])
@pytest.mark.parametrize("H,Hk,dk,dv,lens,states", CASES)
def test_strong_decays(dtype, decay, H, Hk, dk, dv, lens, states):
    r, T, n = gen(H + dk + dv), sum(lens), len(lens)
    x = inputs(r, T, H, Hk, dk, dv, dtype, decay=decay)
    S, dS = (0.3 * r(n, H, dk, dv), 0.3 * r(n, H, dk, dv)) if states else (None, None)
    kw = dict(cu=cu_of(lens), S_in=S)
    saved = binding.chela_gated_delta_fwd(*x[:5], want_saved=True, **kw)[1]
    for s in (saved, None):
        check_dg(binding.chela_gated_delta_bwd(*x, dS_out=dS, saved=s, **kw)[3], x, S, dS, lens, dtype)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("L", [140, 1400])
def test_where_nothing_is_let_through(dtype, L):
    r, H, d = gen(L), 3, 64
    x = inputs(r, L, H, H, d, d, dtype)
    g = x[3]
    t = torch.arange(L, device="cuda")
    g[:, 0] = torch.where(t % 9 == 4, -float("inf"), g[:, 0].float()).to(dtype)
    g[:, 1] = torch.where(t % 40 == 5, torch.finfo(dtype).min, g[:, 1].float()).to(dtype)
    g[:, 2] = torch.where(t % 2 == 0, -300.0, g[:, 2].float()).to(dtype)
    S, dS = r(1, H, d, d), r(1, H, d, d)
    for st, ds in ((S, dS), (None, None), (torch.zeros_like(S), dS)):
        dg = binding.chela_gated_delta_bwd(*x, S_in=st, dS_out=ds)[3]
        assert (dg[g < -256] == 0).all()
        if st is not S:
            assert (dg[0] == 0).all()
        check_dg(dg, x, st, ds, [L], dtype)
