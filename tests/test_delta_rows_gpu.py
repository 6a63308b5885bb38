"""The gated delta rule over runs of several chunks on the GPU, against the definition in 64 bits row by row: a row, an element, a chunk at a run's or a
sequence's end that is lost, stale or another's is found, which a norm over a sequence of thousands of tokens does not show.

Tolerances, before any run.  A rounding to bf16 is off by 2^-8 / sqrt(3) in the root of the mean of squares at most (evenly within half a step), and an output in bf16 has at
most nine on its way, itself among them (test_delta_gpu): sigma = 2^-8 sqrt(9 / 3) of a row's own size.  In fp32 sigma = 4 sqrt(12 128) 2^-24, as there.  A chunk as a whole may be
off by sigma of its norm (or of that of the sequence's chunks on average, where it is smaller: what is rounded on the way need not be smaller with it), an element by 8 sigma of
what the elements of its row are, or of those of its chunk: of the 2e6 elements of the largest case none is expected beyond 6.
dg and dbeta are one number a token, a sum of n terms of either sign whose independent errors, sigma t_i each, leave sigma sqrt(sum t_i^2): as much as sigma of the number
itself in the mean over many, since its square is sum t_i^2 in the mean, but any multiple of it where the number is small by chance.  A sum of m such squares is below a
quarter of its mean with a probability of 1e-3 at m = 16 (chi squared), so a last chunk of fewer rows counts with the one in front of it."""
import numpy as np
import pytest
import torch

from oracle import delta as R
from paper_2406_08128_amd import binding
from test_delta_gpu import BF, DTYPES, MANY, RUNS, cu_of, f64, gen, inputs, offsets

pytestmark = pytest.mark.gpu
SIGMA = {torch.bfloat16: 2.0 ** -8 * 3 ** 0.5, torch.float32: 4 * np.sqrt(12 * 128) * 2.0 ** -24}


def row_by_row(what, got, ref, chunk, elements=True):
    """got, ref [L, width] (or [L]: by chunks alone), rows of one sequence from its first one on."""
    L, sigma = len(ref), SIGMA[got.dtype]
    g = f64(got)
    assert np.isfinite(g).all(), what
    off, ref = (x.reshape(L, -1) for x in (g - ref, ref))
    starts = np.arange(0, L, chunk)
    if not elements and 0 < L % chunk < MANY:
        starts = starts[:-1]
    sums = lambda x: np.add.reduceat((x ** 2).sum(1), starts)  # noqa: E731
    size, n = sums(ref), np.diff(np.append(starts, L))
    mean = size / n / ref.shape[1]                                                  # of an element of the chunk, squared
    over = np.maximum(size, n * (size.sum() / L))
    worst = np.sqrt(sums(off) / over)
    assert (worst <= sigma).all(), (what, "chunk", int(worst.argmax()), float(worst.max()), sigma)
    if elements:
        own = np.sqrt(np.maximum((ref ** 2).mean(1), np.repeat(mean, n)))[:, None]
        at = np.abs(off) / own
        assert (at <= 8 * sigma).all(), (what, "element", np.unravel_index(int(at.argmax()), at.shape), float(at.max()), 8 * sigma)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("states", [False, True])
@pytest.mark.parametrize("H,Hk,dk,dv,lens", RUNS)
def test_rows_of_runs(dtype, states, H, Hk, dk, dv, lens):
    r, T, n = gen(dk + 2 * dv + len(lens)), sum(lens), len(lens)
    x = inputs(r, T, H, Hk, dk, dv, dtype, decay=4.0)
    S, dS = (0.3 * r(n, H, dk, dv), 0.3 * r(n, H, dk, dv)) if states else (None, None)
    kw = dict(scale=0.1, cu=cu_of(lens), S_in=S)
    S_out = torch.empty(n, H, dk, dv, device="cuda") if states else None
    O0 = binding.chela_gated_delta_fwd(*x[:5], S_out=S_out, **kw)[0]
    O1, saved = binding.chela_gated_delta_fwd(*x[:5], S_out=S_out, want_saved=True, **kw)
    ways = [binding.chela_gated_delta_bwd(*x[:5], x[5], dS_out=dS, saved=s, **kw) for s in (saved, None)]
    q, k, v, g, beta, dO = (f64(t) for t in x)
    chunk, share = 64 if dtype == BF else 32, H // Hk
    for i, (a, b) in enumerate(zip(offsets(lens), offsets(lens)[1:])):
        if b - a < 2 * chunk:
            continue
        sums = np.zeros((2, b - a, Hk, dk))
        for h in range(H):
            args = (q[a:b, h // share], k[a:b, h // share], v[a:b, h], g[a:b, h], beta[a:b, h])
            st, ds = (None, None) if S is None else (f64(S[i, h]), f64(dS[i, h]))
            O = R.delta_fwd(*args, 0.1, st)[0]
            ref = R.delta_bwd(*args, dO[a:b, h], 0.1, st, ds)
            for t in (O0, O1):
                row_by_row(("O", i, h), t[a:b, h], O, chunk)
            for d in ways:
                row_by_row(("dV", i, h), d[2][a:b, h], ref["dV"], chunk)
                row_by_row(("dg", i, h), d[3][a:b, h], ref["dg"], chunk, elements=False)
                row_by_row(("dbeta", i, h), d[4][a:b, h], ref["dbeta"], chunk, elements=False)
            sums[0, :, h // share] += ref["dQ"]
            sums[1, :, h // share] += ref["dK"]
        for h in range(Hk):
            for d in ways:
                for m, name in enumerate(("dQ", "dK")):
                    row_by_row((name, i, h), d[m][a:b, h], sums[m, :, h], chunk)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("H,Hk,dk,dv,L,piece", [(2, 1, 64, 64, 4200, 1024), (1, 1, 128, 128, 2305, 512), (1, 1, 64, 128, 8300, 512)])
def test_runs_and_pieces_short_enough_to_go_chunk_by_chunk(dtype, H, Hk, dk, dv, L, piece):
    # the same sequence in pieces, each from the state that the one in front left: other kernels, the same rows
    if dtype != BF and dk + dv == 128:
        piece = 1024                                             # (32 chunks of 32; 8 of them with heads of 128)
    elif dtype != BF:
        piece = 256
    r = gen(L)
    x = inputs(r, L, H, Hk, dk, dv, dtype, decay=4.0)[:5]
    whole_S, S = torch.empty(1, H, dk, dv, device="cuda"), torch.zeros(1, H, dk, dv, device="cuda")
    whole = binding.chela_gated_delta_fwd(*x, S_out=whole_S)[0]
    parts = torch.cat([binding.chela_gated_delta_fwd(*(t[a:a + piece] for t in x), S_in=S, S_out=S)[0] for a in range(0, L, piece)])
    for h in range(H):
        row_by_row(("O", h), whole[:, h], f64(parts[:, h]), 64 if dtype == BF else 32)
    # a state has six roundings of two parts on its way, in either (test_delta_gpu)
    rel = 4 * np.sqrt(12 * 128) * 2.0 ** -24 + (2.0 ** -16 * 6 ** 0.5 if dtype == BF else 0)
    assert (whole_S - S).double().norm() <= 2 * rel * S.double().norm()
