"""Layer norm of rows far from zero, on the GPU: the squares are of what is left without the mean.

Tolerance, before any run.  x - m is exact where x is within a factor of two of the mean m as rounded (Sterbenz), whatever m is off by; that comes off every
element alike and goes again with the mean of what is left.  So n is as good as for rows about zero of the same spread: the masses of oracle.delta.layer_norm_fwd and
_bwd on the centred rows, D + 64 roundings of 2^-24 of them.  m itself is off by at most 40 roundings of its own size (a thread adds up to 17 elements, then 6
steps over a wave and up to 8 waves, one product), and the sum of squares taken about it is larger by that squared over the variance, which is taken off again: its
roundings count for as much more.
tests/test_layer_norm_far_host.py shows that this tells rows of zeros, of the other sign, and of a variance taken as E x^2 - m^2."""
import numpy as np
import pytest
import torch

from oracle import delta as R
from paper_2406_08128_amd import binding
from test_delta_gpu import BF, F32, HALF, f64, gen

pytestmark = pytest.mark.gpu


def far_tolerance(mass, ref, c, D, far, half, extra=0):
    """c: the centred rows; far: the size of the mean."""
    more = 1 + (40 * 2.0 ** -24 * far) ** 2 / (c ** 2).mean(-1, keepdims=True)
    return (D + 64 + extra) * 2.0 ** -24 * mass * (more if mass.ndim == c.ndim else more.max()) + half * np.abs(ref)


def far_rows(r, rows, D, far, spread):
    return far + spread * r(rows, D)


FAR = [(20, 768, 1000.0, 0.01), (20, 513, 1000.0, 0.01), (7, 1531, -1000.0, 0.02), (5, 4096, 300.0, 0.01), (3, 8191, 100.0, 0.01), (9, 64, 4096.0, 0.05)]


def close(what, got, ref, tol):
    off = np.abs(f64(got) - ref)
    assert np.isfinite(f64(got)).all() and (off <= tol).all(), (what, float((off / tol).max()))


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("rows,D,far,spread", FAR)
def test_rows_far_from_zero(dtype, rows, D, far, spread):
    # (dtype: of the block's output and of N; the stream is fp32)
    r, eps = gen(D), 0.0
    X, w, b = far_rows(r, rows, D, far, spread), 1 + 0.3 * r(D), r(D)
    dN, up = r(rows, D).to(dtype), r(rows, D)
    x, half = f64(X), HALF[dtype]
    c = x - x.mean(-1, keepdims=True)
    v, m = R.layer_norm_fwd(c, None, f64(w), f64(b), eps)
    N = torch.empty(rows, D, dtype=dtype, device="cuda")
    after, got = binding.chela_layer_norm_fwd(X, w=w, b=b, Nrm=N, eps=eps)
    assert after is X and got is N
    close("N", N, v["N"], far_tolerance(m["N"], v["N"], c, D, far, half))
    for u in (None, up):
        dX, dw, db = binding.chela_layer_norm_bwd(X, dN, w=w, want_db=True, dX_out=u, eps=eps)
        v, m = R.layer_norm_bwd(c, f64(dN), f64(w), f64(u), eps)
        close("dX", dX, v["dX"], far_tolerance(m["dX"], v["dX"], c, D, far, HALF[F32]))
        close("dw", dw, v["dw"], far_tolerance(m["dw"], v["dw"], c, D, far, HALF[F32], rows))
        close("db", db, v["db"], (rows + 64) * 2.0 ** -24 * m["db"] + HALF[F32] * np.abs(v["db"]))


@pytest.mark.parametrize("D", [768, 1531])
def test_a_residual_that_is_added_far_from_zero(D):
    # X + Y is rounded to fp32 as it is stored, and N is of the sum as the thread has it: the same
    r, rows = gen(D + 1), 11
    X, Y = far_rows(r, rows, D, 1000.0, 0.01), (0.01 * r(rows, D)).to(BF)
    after, N = binding.chela_layer_norm_fwd(X, Y=Y, eps=0.0)
    assert torch.equal(after, X + Y.float())
    x = f64(after)
    c = x - x.mean(-1, keepdims=True)
    v, m = R.layer_norm_fwd(c, eps=0.0)
    close("N", N, v["N"], far_tolerance(m["N"], v["N"], c, D, 1000.0, HALF[BF]))
