"""Operators on rows on the GPU, element by element against their definitions in 64 bits (oracle/rows.py).

Tolerances, before any run: an output element may be off by half a step of its type (bf16 2^-8, fp32 2^-24, relative) and by n 2^-24 of its
mass, the same sum over magnitudes, where n bounds the fp32 roundings in a row that a term goes through:
  convolution      8 taps' products and sums, the activation (its exponential's argument is off by |u| 2^-24, u of a few): n = 64
  scan             per row a term's decay is rounded, exponentiated (argument of a few: 6 steps) and multiplied in: 8 a row, and the sum
                   over at most 32 states and the activations: n = 8 L + 128 for a sequence of L rows, and as many again for a gradient
  sums over rows   one rounding per row on top: + T
  norms            the sum of squares over D elements and what follows: n = D + 64
"""
import numpy as np
import pytest
import torch

from oracle import rows as R
from paper_2406_08128_amd import binding

pytestmark = pytest.mark.gpu

HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
BF, F32 = torch.bfloat16, torch.float32
DTYPES = [BF, F32]


def f64(t):
    return t.detach().double().cpu().numpy()


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return lambda *s: torch.randn(*s, generator=g, device="cuda")


def check(name, got, ref, mass, n):
    tol = R.tolerance(ref, mass, n, HALF[got.dtype])
    off = np.abs(f64(got) - ref)
    assert np.isfinite(f64(got)).all(), name
    worst = float((off / tol).max()) if off.size else 0.0
    assert worst <= 1.0, (name, worst, np.unravel_index(int((off / tol).argmax()), off.shape))


def same(a, b):
    return (a is None) == (b is None) and (a is None or torch.equal(a, b))


def offsets(lens, first=0):
    return np.concatenate([[first], first + np.cumsum(lens)]).astype(np.int64)


def cu_of(lens, first=0):
    return torch.tensor(offsets(lens, first), dtype=torch.int32, device="cuda")


def wide_rows(t, extra=3):
    """The same rows as a slice of wider ones, off 16-byte boundaries."""
    w = torch.full((*t.shape[:-1], t.shape[-1] + extra), float("nan"), dtype=t.dtype, device=t.device)
    w[..., 1:1 + t.shape[-1]] = t
    return w[..., 1:1 + t.shape[-1]]


# ------------------------------------------------------------------------------------------- short causal convolution
CONV = [  # m, D, lengths, states, bias, silu, strided
    (4, 64, [1], True, True, True, False),
    (4, 64, [16, 32, 48], False, True, True, False),
    (4, 1536, [7, 0, 1, 2, 3, 40, 1], True, True, True, False),
    (3, 200, [33, 65], True, False, True, True),
    (1, 24, [5, 9], False, True, True, False),
    (2, 7, [17, 1, 1, 31], True, True, False, False),
    (5, 1, [70], True, True, True, False),
    (8, 96, [3, 100, 4], True, True, True, False),
    (6, 33, [2, 2, 2, 2], True, False, False, True),
    (7, 2056, [35], False, True, True, False),
]


def conv_reference(X, w, bias, silu, S, dY, dS, lens, first=0):
    o, m = offsets(lens, first), w.shape[1]
    parts = []
    for i in range(len(lens)):
        a, b = o[i], o[i + 1]
        st = None if S is None else S[i]
        y, my, after = R.short_conv_fwd(X[a:b], w, bias, silu, st)
        v, mv = R.short_conv_bwd(X[a:b], w, dY[a:b], bias, silu, st, None if dS is None else dS[i])
        parts.append((y, my, after, v, mv))
    return parts


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,D,lens,states,biased,silu,strided", CONV)
def test_short_conv(dtype, m, D, lens, states, biased, silu, strided):
    r, T, n = gen(D + m), sum(lens), len(lens)
    X, dY = r(T, D).to(dtype), r(T, D).to(dtype)
    w, bias = r(D, m) / m ** 0.5, r(D) if biased else None
    S, dS = (r(n, m - 1, D).to(dtype), r(n, m - 1, D).to(dtype)) if states else (None, None)
    Xs, dYs = (wide_rows(X), wide_rows(dY)) if strided else (X, dY)
    cu = cu_of(lens)
    S_out = torch.full((n, m - 1, D), float("nan"), dtype=dtype, device="cuda")
    Y = binding.chela_short_conv_fwd(Xs, w, bias=bias, silu=silu, cu=cu, S_in=S, S_out=S_out)
    dX, dw, db, dS_in = binding.chela_short_conv_bwd(Xs, w, dYs, bias=bias, silu=silu, cu=cu, S_in=S, dS_out=dS, want_dS_in=True)
    ref = conv_reference(f64(X), f64(w), f64(bias) if biased else None, silu, f64(S) if states else None, f64(dY), f64(dS) if states else None, lens)
    o = offsets(lens)
    for i, (y, my, after, v, mv) in enumerate(ref):
        check("Y", Y[o[i]:o[i + 1]], y, my, 64)
        assert np.array_equal(f64(S_out[i]), after)                     # inputs, as they are
        check("dX", dX[o[i]:o[i + 1]], v["dX"], mv["dX"], 64)
        check("dS_in", dS_in[i], v["dS_in"], mv["dS_in"], 64)
    check("dw", dw, sum(p[3]["dw"] for p in ref), sum(p[4]["dw"] for p in ref), T + 64)
    if biased:
        check("dbias", db, sum(p[3]["dbias"] for p in ref), sum(p[4]["dbias"] for p in ref), T + 64)
    else:
        assert db is None


@pytest.mark.parametrize("dtype", DTYPES)
def test_short_conv_in_place_state_and_equal_lengths(dtype):
    r, m, D, n, L = gen(5), 4, 128, 3, 37
    X, w, S = r(n, L, D).to(dtype), r(D, m), r(n, m - 1, D).to(dtype)
    S2, S_out = S.clone(), torch.empty_like(S)
    a = binding.chela_short_conv_fwd(X, w, S_in=S, S_out=S_out)
    b = binding.chela_short_conv_fwd(X, w, S_in=S2, S_out=S2)
    c = binding.chela_short_conv_fwd(X.view(n * L, D), w, cu=cu_of([L] * n), S_in=S)
    assert torch.equal(a, b) and torch.equal(S_out, S2) and torch.equal(a.view(n * L, D), c)
    # in two pieces, the second from the first's states
    k = 21
    S3 = S.clone()
    p = binding.chela_short_conv_fwd(X[:, :k].contiguous(), w, S_in=S3, S_out=S3)
    q = binding.chela_short_conv_fwd(X[:, k:].contiguous(), w, S_in=S3, S_out=S3)
    assert torch.equal(torch.cat([p, q], 1), a) and torch.equal(S3, S_out)
    # and token by token
    S4 = S.clone()
    for t in range(L):
        y = binding.chela_short_conv_step(X[:, t], w, S4)               # (rows with a stride)
        assert torch.equal(y, a[:, t]), t
    assert torch.equal(S4, S_out)


@pytest.mark.parametrize("D,m", [(64, 4), (7, 4), (1000, 1), (96, 8)])
@pytest.mark.parametrize("dtype", DTYPES)
def test_short_conv_step_against_the_definition(dtype, D, m):
    r, n = gen(9), 5
    x, w, b, S = r(n, D).to(dtype), r(D, m), r(D), r(n, m - 1, D).to(dtype)
    S0 = f64(S)
    y = binding.chela_short_conv_step(x, w, S, bias=b)
    for i in range(n):
        v, mass, after = R.short_conv_fwd(f64(x)[i:i + 1], f64(w), f64(b), True, S0[i])
        check("y", y[i:i + 1], v, mass, 64)
        assert np.array_equal(f64(S[i]), after)


# ------------------------------------------------------------------------------------------- selective scan
SCAN = [  # N, G, D, lengths, states, skip, Z, bias, softplus, strided
    (16, 1, 64, [1], True, True, True, True, True, False),
    (16, 1, 128, [100, 60], True, True, True, True, True, False),
    (16, 2, 136, [9, 0, 1, 2, 40, 16, 15, 17, 1, 64], True, True, True, True, True, False),
    (8, 1, 1, [33], False, False, False, False, True, False),
    (8, 4, 260, [300], True, True, False, True, True, True),
    (32, 1, 65, [31, 70], True, False, True, False, True, False),
    (32, 3, 99, [16, 16, 32], False, True, True, False, False, True),
    (16, 1, 200, [1] * 40, True, True, True, True, True, False),
    (16, 1, 70, [50], True, True, True, True, True, True),
    (16, 5, 5, [50, 20], True, True, True, True, True, False),
]


def scan_inputs(r, T, D, N, G, dtype, softplus=True):
    u, delta, z = r(T, D).to(dtype), r(T, D).to(dtype), r(T, D).to(dtype)
    if not softplus:
        delta = (delta.float().abs() * 0.3).to(dtype)
    both = r(T, 2 * G * N).to(dtype)
    Bm, Cm = both[:, :G * N].unflatten(1, (G, N)), both[:, G * N:].unflatten(1, (G, N))
    return u, delta, z, Bm, Cm, -torch.exp(r(N, D)), r(D), r(D) - 1


def scan_reference(x, S, dY, dS, lens, first=0):
    u, delta, z, Bm, Cm, A, skip, bias, softplus = x
    o, out = offsets(lens, first), []
    cut = lambda t, a, b: None if t is None else t[a:b]  # noqa: E731
    for i in range(len(lens)):
        a, b = o[i], o[i + 1]
        args = (u[a:b], delta[a:b], A, Bm[a:b], Cm[a:b])
        st = None if S is None else S[i]
        f = R.selscan_fwd(*args, skip, cut(z, a, b), bias, softplus, st)
        g = R.selscan_bwd(*args, dY[a:b], skip, cut(z, a, b), bias, softplus, st, None if dS is None else dS[i])
        out.append((f, g))
    return out


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("N,G,D,lens,states,skipped,gated,biased,softplus,strided", SCAN)
def test_selscan(dtype, N, G, D, lens, states, skipped, gated, biased, softplus, strided):
    r, T, n = gen(N + D), sum(lens), len(lens)
    u, delta, z, Bm, Cm, A, skip, bias = scan_inputs(r, T, D, N, G, dtype, softplus)
    dY = r(T, D).to(dtype)
    S, dS = (r(n, N, D), r(n, N, D)) if states else (None, None)
    skip, z, bias = skip if skipped else None, z if gated else None, bias if biased else None
    us, ds, zs, dYs = (wide_rows(t) if strided and t is not None else t for t in (u, delta, z, dY))
    kw = dict(D=skip, Z=zs, delta_bias=bias, softplus=softplus, cu=cu_of(lens), S_in=S)
    S_out = torch.full((n, N, D), float("nan"), device="cuda")
    Y, saved = binding.chela_selscan_fwd(us, ds, A, Bm, Cm, S_out=S_out, want_saved=True, **kw)
    g = binding.chela_selscan_bwd(us, ds, A, Bm, Cm, dYs, dS_out=dS, want_dS_in=True, saved=saved, **kw)
    again = binding.chela_selscan_bwd(us, ds, A, Bm, Cm, dYs, dS_out=dS, want_dS_in=True, **kw)
    assert all([same(a, b) for a, b in zip(g, again)])
    n64 = [None if t is None else f64(t) for t in (u, delta, z, Bm, Cm, A, skip, bias)]
    ref = scan_reference((*n64, softplus), f64(S) if states else None, f64(dY), f64(dS) if states else None, lens)
    o, longest = offsets(lens), max(lens)
    k = 8 * longest + 128
    names = ("dU", "ddelta", "dA", "dB", "dC", "dD", "dZ", "dbias", "dS_in")
    got = dict(zip(names, g))
    for i, ((f, mf), (v, mv)) in enumerate(ref):
        rows = slice(o[i], o[i + 1])
        check("Y", Y[rows], f["Y"], mf["Y"], k)
        check("S_out", S_out[i], f["S_out"], mf["S_out"], k)
        for name in ("dU", "ddelta", "dB", "dC"):
            check(name, got[name][rows], v[name], mv[name], 2 * k + D)
        if gated:
            check("dZ", got["dZ"][rows], v["dZ"], mv["dZ"], 2 * k)
        check("dS_in", got["dS_in"][i], v["dS_in"], mv["dS_in"], 2 * k)
    for name, there in (("dA", True), ("dD", skipped), ("dbias", biased)):
        if there:
            check(name, got[name], sum(p[1][0][name] for p in ref), sum(p[1][1][name] for p in ref), 2 * k + T)
        else:
            assert got[name] is None
    assert gated or got["dZ"] is None


@pytest.mark.parametrize("dtype", DTYPES)
def test_selscan_many_chunks_pieces_and_single_tokens(dtype):
    # long enough to be cut into many chunks; in pieces and token by token the states carry over
    r, D, N, n, L = gen(11), 96, 16, 2, 700
    u, delta, z, Bm, Cm, A, skip, bias = scan_inputs(r, n * L, D, N, 1, dtype)
    S = r(n, N, D)
    v3 = lambda t: t.reshape(n, L, *t.shape[1:])  # noqa: E731
    u, delta, z, Bm, Cm = (v3(t) for t in (u, delta, z, Bm, Cm))
    kw = dict(D=skip, delta_bias=bias)
    S_out = torch.empty_like(S)
    Y, _ = binding.chela_selscan_fwd(u, delta, A, Bm, Cm, Z=z, S_in=S, S_out=S_out, **kw)
    # the same buffer in front and behind
    S2 = S.clone()
    Y2, _ = binding.chela_selscan_fwd(u, delta, A, Bm, Cm, Z=z, S_in=S2, S_out=S2, **kw)
    assert torch.equal(Y, Y2) and torch.equal(S_out, S2)
    n64 = [f64(t) for t in (u, delta, z, Bm, Cm, A, skip, bias)]
    for i in range(n):
        f, mf = R.selscan_fwd(n64[0][i], n64[1][i], n64[5], n64[3][i], n64[4][i], n64[6], n64[2][i], n64[7], True, f64(S)[i])
        check("Y", Y[i], f["Y"], mf["Y"], 8 * L + 128)
        check("S_out", S_out[i], f["S_out"], mf["S_out"], 8 * L + 128)
    # pieces of odd lengths, then single tokens
    S3, got, t = S.clone(), [], 0
    for k in (1, 130, 301, 17, 201):
        c = [x[:, t:t + k].contiguous() for x in (u, delta, z, Bm, Cm)]
        got.append(binding.chela_selscan_fwd(c[0], c[1], A, c[3], c[4], Z=c[2], S_in=S3, S_out=S3, **kw)[0])
        t += k
    for t in range(t, L):
        got.append(binding.chela_selscan_step(u[:, t], delta[:, t], A, Bm[:, t], Cm[:, t], S3, z=z[:, t], **kw)[:, None])
    got = torch.cat(got, 1)
    for i in range(n):
        f, mf = R.selscan_fwd(n64[0][i], n64[1][i], n64[5], n64[3][i], n64[4][i], n64[6], n64[2][i], n64[7], True, f64(S)[i])
        check("Y", got[i], f["Y"], mf["Y"], 8 * L + 128)
        check("S_out", S3[i], f["S_out"], mf["S_out"], 8 * L + 128)


@pytest.mark.parametrize("lens", [[6700], [2300, 0, 4400]])
def test_selscan_hundreds_of_chunks(lens):
    # (so many that the carries take several rounds)
    r, D, N, T, n = gen(89), 8, 8, sum(lens), len(lens)
    u, delta, z, Bm, Cm, A, skip, bias = scan_inputs(r, T, D, N, 1, F32)
    dY, S, dS = r(T, D), r(n, N, D), r(n, N, D)
    kw = dict(D=skip, Z=z, delta_bias=bias - 3, cu=cu_of(lens), S_in=S)          # (steps small enough for states to last through chunks)
    S_out = torch.empty_like(S)
    Y, saved = binding.chela_selscan_fwd(u, delta, A, Bm, Cm, S_out=S_out, want_saved=True, **kw)
    g = dict(zip(("dU", "ddelta", "dA", "dB", "dC", "dD", "dZ", "dbias", "dS_in"),
                 binding.chela_selscan_bwd(u, delta, A, Bm, Cm, dY, dS_out=dS, want_dS_in=True, saved=saved, **kw)))
    n64 = [f64(t) for t in (u, delta, z, Bm, Cm, A, skip, bias - 3)]
    o, k = offsets(lens), 8 * max(lens) + 128
    ref = scan_reference((*n64, True), f64(S), f64(dY), f64(dS), lens)
    for i, ((f, mf), (v, mv)) in enumerate(ref):
        rows = slice(o[i], o[i + 1])
        check("Y", Y[rows], f["Y"], mf["Y"], k)
        check("S_out", S_out[i], f["S_out"], mf["S_out"], k)
        for name in ("dU", "ddelta", "dB", "dC", "dZ"):
            check(name, g[name][rows], v[name], mv[name], 2 * k + D)
        check("dS_in", g["dS_in"][i], v["dS_in"], mv["dS_in"], 2 * k)
    for name in ("dA", "dD", "dbias"):
        check(name, g[name], sum(p[1][0][name] for p in ref), sum(p[1][1][name] for p in ref), 2 * k + T)


@pytest.mark.parametrize("lasting", [False, True])
@pytest.mark.parametrize("N,G,D,lens", [(8, 1, 8, [6700]), (8, 1, 8, [2300, 0, 4400]), (16, 2, 24, [3000]), (32, 1, 65, [700, 1900])])
def test_selscan_chunks_hand_on_all_digits(N, G, D, lens, lasting):
    # every term held to the roundings of the rows that it has passed (a carry in 16 bits is off by ten times that, see the host's tests)
    r, T, n = gen(103 + N), sum(lens), len(lens)
    u, delta, z, Bm, Cm, A, skip, bias = scan_inputs(r, T, D, N, G, F32)
    bias = bias - 3
    A = A / 64 if lasting else A                                        # (states that last for thousands of rows, or for tens)
    dY, S, dS = r(T, D), r(n, N, D), r(n, N, D)
    kw = dict(D=skip, Z=z, delta_bias=bias, cu=cu_of(lens), S_in=S)
    S_out = torch.empty_like(S)
    Y, saved = binding.chela_selscan_fwd(u, delta, A, Bm, Cm, S_out=S_out, want_saved=True, **kw)
    g = dict(zip(("dU", "ddelta", "dA", "dB", "dC", "dD", "dZ", "dbias", "dS_in"),
                 binding.chela_selscan_bwd(u, delta, A, Bm, Cm, dY, dS_out=dS, want_dS_in=True, saved=saved, **kw)))
    n64 = [f64(t) for t in (u, delta, z, Bm, Cm, A, skip, bias)]
    o = offsets(lens)
    ref = scan_reference((*n64, True), f64(S), f64(dY), f64(dS), lens)
    for i, ((f, _), (v, _)) in enumerate(ref):
        rows = slice(o[i], o[i + 1])
        k = R.selscan_roundings(n64[0][rows], n64[1][rows], n64[5], n64[3][rows], n64[4][rows], f64(dY)[rows], n64[6], n64[2][rows], n64[7], True,
                                f64(S)[i], f64(dS)[i])
        check("Y", Y[rows], f["Y"], k["Y"], 1)
        check("S_out", S_out[i], f["S_out"], k["S_out"], 1)
        for name in ("dU", "ddelta", "dB", "dC", "dZ"):
            check(name, g[name][rows], v[name], k[name], 1)
        check("dS_in", g["dS_in"][i], v["dS_in"], k["dS_in"], 1)


@pytest.mark.parametrize("N,G,D", [(16, 1, 64), (8, 2, 30), (32, 1, 200), (16, 4, 1000)])
@pytest.mark.parametrize("dtype", DTYPES)
def test_selscan_step_against_the_definition(dtype, N, G, D):
    r, n = gen(13), 4
    u, delta, z, Bm, Cm, A, skip, bias = scan_inputs(r, n, D, N, G, dtype)
    S = r(n, N, D)
    S0 = f64(S)
    y = binding.chela_selscan_step(u, delta, A, Bm, Cm, S, D=skip, z=z, delta_bias=bias)
    for i in range(n):
        one = [f64(t)[i:i + 1] for t in (u, delta, Bm, Cm, z)]
        v, m = R.selscan_fwd(one[0], one[1], f64(A), one[2], one[3], f64(skip), one[4], f64(bias), True, S0[i])
        check("y", y[i:i + 1], v["Y"], m["Y"], 136)
        check("S", S[i], v["S_out"], m["S_out"], 136)


# ------------------------------------------------------------------------------------------- pools of states, rows of nobody
@pytest.mark.parametrize("dtype", DTYPES)
def test_slots_and_rows_of_nobody(dtype):
    r, m, D, N = gen(17), 4, 72, 16
    lens, first, T = [5, 0, 40, 1, 90], 3, 150                     # rows 0 .. 2 and 139 .. 149 are nobody's
    cu, n = cu_of(lens, first), len(lens)
    o = offsets(lens, first)
    slots = torch.tensor([6, 2, -1, 0, 99], dtype=torch.int32, device="cuda")        # a pool of 8; sequences 2 and 4 have no state
    u, delta, z, Bm, Cm, A, skip, bias = scan_inputs(r, T, D, N, 1, dtype)
    dY, w = r(T, D).to(dtype), r(D, m)
    owned = np.zeros(T, bool)
    owned[o[0]:o[-1]] = True
    bad = torch.tensor(~owned, device="cuda")
    for t in (u, delta, z, Bm, Cm, dY):
        t[bad] = float("nan")                                      # nothing of these rows is taken in
    mark = 12345.0
    pool, conv_pool = r(8, N, D), r(8, m - 1, D).to(dtype)
    p0, c0 = pool.clone(), conv_pool.clone()
    Y = torch.full((T, D), mark, dtype=dtype, device="cuda")
    kw = dict(D=skip, Z=z, delta_bias=bias, cu=cu)
    binding.chela_selscan_fwd(u, delta, A, Bm, Cm, S_in=pool, S_out=pool, slots=slots, Y=Y, **kw)
    Yc = torch.full((T, D), mark, dtype=dtype, device="cuda")
    binding.chela_short_conv_fwd(u, w, cu=cu, S_in=conv_pool, S_out=conv_pool, slots=slots, Y=Yc)
    assert (Y[bad].float() == Y.new_tensor(mark).float()).all() and (Yc[bad].float() == Y.new_tensor(mark).float()).all()
    where = {0: 6, 1: 2, 3: 0}
    n64 = [f64(t) for t in (u, delta, z, Bm, Cm, A, skip, bias)]
    for i in range(n):
        a, b = o[i], o[i + 1]
        st = f64(p0)[where[i]] if i in where else None
        f, mf = R.selscan_fwd(n64[0][a:b], n64[1][a:b], n64[5], n64[3][a:b], n64[4][a:b], n64[6], n64[2][a:b], n64[7], True, st)
        check("Y", Y[a:b], f["Y"], mf["Y"], 8 * 90 + 128)
        y, my, after = R.short_conv_fwd(n64[0][a:b], f64(w), None, True, f64(c0)[where[i]] if i in where else None)
        check("Yc", Yc[a:b], y, my, 64)
        if i in where:
            check("S", pool[where[i]], f["S_out"], mf["S_out"], 8 * 90 + 128)
            assert np.array_equal(f64(conv_pool[where[i]]), after)
    for k in range(8):
        if k not in where.values():
            assert torch.equal(pool[k], p0[k]) and torch.equal(conv_pool[k], c0[k])
    # gradients: rows of nobody keep what the buffers hold (allocated by the call: only that they take in nothing is seen)
    g = binding.chela_selscan_bwd(u, delta, A, Bm, Cm, dY, want_dS_in=True, **kw)
    h = binding.chela_short_conv_bwd(u, w, dY, cu=cu, want_dS_in=True)
    for t in (g[2], g[5], g[7], g[8], h[1], h[3]):
        assert torch.isfinite(t).all()
    ok = torch.tensor(owned, device="cuda")
    for t in (*g[:2], g[3], g[4], g[6], h[0]):
        assert torch.isfinite(t[ok].float()).all()
    # single tokens: rows without a slot stay
    y = torch.full((n, D), mark, dtype=dtype, device="cuda")
    yc = y.clone()
    before, cbefore = pool.clone(), conv_pool.clone()
    x = [t[ok][:n].contiguous() for t in (u, delta, z, Bm, Cm)]
    binding.chela_selscan_step(x[0], x[1], A, x[3], x[4], pool, D=skip, z=x[2], delta_bias=bias, slots=slots, y=y)
    binding.chela_short_conv_step(x[0], w, conv_pool, slots=slots, y=yc)
    for i in range(n):
        if i in where:
            assert not torch.equal(pool[where[i]], before[where[i]]) and (y[i].float() != y.new_tensor(mark).float()).any()
        else:
            assert (y[i] == y.new_tensor(mark)).all() and (yc[i] == y.new_tensor(mark)).all()
    for k in range(8):
        if k not in where.values():
            assert torch.equal(pool[k], before[k]) and torch.equal(conv_pool[k], cbefore[k])


def poisoned(*shapes):
    """What the allocator gives out next, for tensors of these (shape, dtype), holds no numbers."""
    torch.cuda.synchronize()
    held = [torch.full(s, float("nan"), dtype=t, device="cuda") for s, t in shapes for _ in range(8)]
    torch.cuda.synchronize()
    del held


@pytest.mark.parametrize("named", [False, True])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("lens,first,T", [([5, 0, 40, 1, 90], 3, 150), ([33, 7], 0, 1000), ([20], 901, 930), ([], 4, 70), ([0, 0], 0, 61)])
def test_rows_of_nobody_are_zero_in_new_outputs(lens, first, T, dtype, named):
    # (named: with a stream named a call goes through the binding's own lines, else through the compiled host path)
    r, m, D, N, n = gen(101 + T), 4, 72, 16, len(lens)
    kw = dict(stream=torch.cuda.current_stream()) if named else {}
    cu = cu_of(lens, first)
    owned = np.zeros(T, bool)
    owned[first:first + sum(lens)] = True
    own, bad = torch.tensor(owned, device="cuda"), torch.tensor(~owned, device="cuda")
    u, delta, z, Bm, Cm, A, skip, bias = scan_inputs(r, T, D, N, 1, dtype)
    dY, w = r(T, D).to(dtype), r(D, m)
    for t in (u, delta, z, Bm, Cm, dY):
        t[bad] = float("nan")
    scan = dict(D=skip, Z=z, delta_bias=bias, cu=cu, **kw)
    rows, maps = ((T, D), dtype), ((T, 1, N), dtype)
    for run, new, given in (
            (lambda **k: binding.chela_short_conv_fwd(u, w, cu=cu, **kw, **k), [rows], True),
            (lambda **k: binding.chela_short_conv_fwd(wide_rows(u), w[:, :1].contiguous(), cu=cu, **kw, **k), [rows], True),
            (lambda **k: binding.chela_selscan_fwd(u, delta, A, Bm, Cm, **scan, **k)[0], [rows], True),
            (lambda: binding.chela_short_conv_bwd(u, w, dY, cu=cu, **kw)[:1], [rows], False),
            (lambda: binding.chela_short_conv_bwd(u[:, :71], w[:71], dY[:, :71], cu=cu, **kw)[:1], [((T, 71), dtype)], False),
            (lambda: [binding.chela_selscan_bwd(u, delta, A, Bm, Cm, dY, **scan)[k] for k in (0, 1, 3, 4, 6)], [rows, maps], False),
            (lambda: [binding.chela_selscan_bwd(u, delta, A, Bm, Cm, dY, cu=cu, **kw)[k] for k in (0, 1, 3, 4)], [rows, maps], False)):
        poisoned(*new)
        got = run()
        for t in (got,) if given else got:
            assert (t[bad] == 0).all() and torch.isfinite(t).all()
        if given:                                                        # one that the caller has keeps its rows
            Y = torch.full((T, D), 7.0, dtype=dtype, device="cuda")
            assert run(Y=Y) is Y and (Y[bad] == 7).all() and torch.equal(Y[own], got[own])
    # single tokens: requests without a state
    R, slots = 5, torch.tensor([2, -1, 0, 7, 4], dtype=torch.int32, device="cuda")
    u, delta, z, Bm, Cm, A, skip, bias = scan_inputs(r, R, D, N, 1, dtype)
    S, C = r(5, N, D), r(5, m - 1, D).to(dtype)
    for run in (lambda **k: binding.chela_selscan_step(u, delta, A, Bm, Cm, S.clone(), z=z, slots=slots, **kw, **k),
                lambda **k: binding.chela_short_conv_step(u, w, C.clone(), slots=slots, **kw, **k),
                lambda **k: binding.chela_short_conv_step(wide_rows(u), w, C.clone(), slots=slots, **kw, **k)):
        poisoned(((R, D), dtype))
        y = run()
        mine, none = [0, 2, 4], [1, 3]
        assert (y[none] == 0).all() and torch.isfinite(y).all()
        y2 = torch.full((R, D), 7.0, dtype=dtype, device="cuda")
        assert run(y=y2) is y2 and (y2[none] == 7).all() and torch.equal(y2[mine], y[mine])


@pytest.mark.parametrize("n", [70, 300, 5000])
def test_many_sequences(n):
    # more of them than lanes, than 64 lanes' steps; short ones, many without rows, at the ends too
    r, rng, D, N, m = gen(53), np.random.default_rng(n), 24, 8, 4
    lens = rng.integers(0, 5, n) * rng.integers(0, 2, n)
    lens[:3] = lens[-2:] = 0
    first = 2
    T, o = int(lens.sum()) + first + 3, offsets(lens, first)
    cu = cu_of(lens, first)
    u, delta, z, Bm, Cm, A, skip, bias = scan_inputs(r, T, D, N, 1, F32)
    dY, w, S, dS = r(T, D), r(D, m), r(n, N, D), r(n, N, D)
    C, dC = r(n, m - 1, D), r(n, m - 1, D)
    kw = dict(D=skip, Z=z, delta_bias=bias, cu=cu)
    S_out, C_out = torch.full_like(S, float("nan")), torch.full_like(C, float("nan"))
    Y, saved = binding.chela_selscan_fwd(u, delta, A, Bm, Cm, S_in=S, S_out=S_out, want_saved=True, **kw)
    S2 = S.clone()
    Y2, _ = binding.chela_selscan_fwd(u, delta, A, Bm, Cm, S_in=S2, S_out=S2, **kw)
    owned = slice(int(o[0]), int(o[-1]))
    assert torch.equal(Y[owned], Y2[owned]) and torch.equal(S_out, S2)
    g = binding.chela_selscan_bwd(u, delta, A, Bm, Cm, dY, S_in=S, dS_out=dS, want_dS_in=True, saved=saved, **kw)
    y = binding.chela_short_conv_fwd(u, w, cu=cu, S_in=C, S_out=C_out)
    h = binding.chela_short_conv_bwd(u, w, dY, cu=cu, S_in=C, dS_out=dC, want_dS_in=True)
    n64 = [f64(t) for t in (u, delta, z, Bm, Cm, A, skip, bias)]
    ref = scan_reference((*n64, True), f64(S), f64(dY), f64(dS), lens, first)
    cref = conv_reference(n64[0], f64(w), None, True, f64(C), f64(dY), f64(dC), lens, first)
    k = 8 * 4 + 128
    cat = lambda parts, rows: np.concatenate(parts) if rows else np.stack(parts)  # noqa: E731
    for name, got, rows in (("Y", Y[owned], True), ("S_out", S_out, False)):
        check(name, got, cat([p[0][0][name] for p in ref], rows), cat([p[0][1][name] for p in ref], rows), k)
    got = dict(zip(("dU", "ddelta", "dA", "dB", "dC", "dD", "dZ", "dbias", "dS_in"), g))
    for name in ("dU", "ddelta", "dB", "dC", "dZ"):
        check(name, got[name][owned], cat([p[1][0][name] for p in ref], True), cat([p[1][1][name] for p in ref], True), 2 * k + D)
    check("dS_in", got["dS_in"], cat([p[1][0]["dS_in"] for p in ref], False), cat([p[1][1]["dS_in"] for p in ref], False), 2 * k)
    for name in ("dA", "dD", "dbias"):
        check(name, got[name], sum(p[1][0][name] for p in ref), sum(p[1][1][name] for p in ref), 2 * k + T)
    check("y", y[owned], cat([p[0] for p in cref], True), cat([p[1] for p in cref], True), 64)
    assert np.array_equal(f64(C_out), cat([p[2] for p in cref], False))
    check("dX", h[0][owned], cat([p[3]["dX"] for p in cref], True), cat([p[4]["dX"] for p in cref], True), 64)
    check("conv dS_in", h[3], cat([p[3]["dS_in"] for p in cref], False), cat([p[4]["dS_in"] for p in cref], False), 64)
    check("dw", h[1], sum(p[3]["dw"] for p in cref), sum(p[4]["dw"] for p in cref), T + 64)


def test_no_rows():
    D, N, m = 64, 16, 4
    S, C = torch.randn(2, N, D, device="cuda"), torch.randn(2, m - 1, D, device="cuda")
    x, B = torch.empty(0, D, device="cuda"), torch.empty(0, N, device="cuda")
    cu = torch.zeros(3, dtype=torch.int32, device="cuda")
    S_out, C_out = torch.full_like(S, 7.0), torch.full_like(C, 7.0)
    A, w = -torch.ones(N, D, device="cuda"), torch.ones(D, m, device="cuda")
    binding.chela_selscan_fwd(x, x, A, B, B, cu=cu, S_in=S, S_out=S_out)
    binding.chela_short_conv_fwd(x, w, cu=cu, S_in=C, S_out=C_out)
    assert torch.equal(S, S_out) and torch.equal(C, C_out)
    g = binding.chela_selscan_bwd(x, x, A, B, B, x, D=torch.ones(D, device="cuda"), cu=cu, dS_out=S, want_dS_in=True)
    assert (g[2] == 0).all() and (g[5] == 0).all() and torch.equal(g[8], S)
    h = binding.chela_short_conv_bwd(x, w, x, bias=torch.ones(D, device="cuda"), cu=cu, dS_out=C, want_dS_in=True)
    assert (h[1] == 0).all() and (h[2] == 0).all() and torch.equal(h[3], C)
    n = binding.chela_block_norm_bwd(x, x, x, x, w_post=torch.ones(D, device="cuda"), w_pre=torch.ones(D, device="cuda"))
    assert (n[3] == 0).all() and (n[4] == 0).all()


@pytest.mark.parametrize("sfx,dtype", [("", BF), ("_f32", F32)])
@pytest.mark.parametrize("T,packed", [(0, False), (0, True), (9, True)])
def test_no_sequences(sfx, dtype, T, packed):
    # addresses of states all the same, as a caller from C may hand them over: there is nothing to pass on, and no error
    L, D, N, m, st = binding.lib(), 64, 16, 4, torch.cuda.current_stream().cuda_stream
    cu = torch.zeros(1, dtype=torch.int32, device="cuda")
    pcu = cu.data_ptr() if packed else None
    X, dX, dZ = (torch.full((9, D), 3.0, dtype=dtype, device="cuda") for _ in range(3))
    Bm, dB, dC = (torch.full((9, N), 3.0, dtype=dtype, device="cuda") for _ in range(3))
    w, dw, A, dA, b, db = (torch.full(s, 3.0, device="cuda") for s in ((D, m), (D, m), (N, D), (N, D), (D,), (D,)))
    S, C, S2, C2 = (torch.full(s, 5.0, dtype=t, device="cuda") for s, t in ((((1, N, D)), F32), ((1, m - 1, D), dtype)) * 2)
    x, p = X.data_ptr(), lambda t: t.data_ptr()  # noqa: E731
    conv = (x, D, p(w), m, p(b), 1, pcu, 0, T, D)
    scan = (x, D, x, D, p(A), p(Bm), N, p(Bm), N, None, None, 0, None, 1, pcu, 0, T, D, N, 1)
    assert getattr(L, "chela_short_conv_bwd" + sfx)(*conv, p(C), x, D, p(C), p(dX), p(dw), p(db), p(C2), st) == 0
    assert (dw == 0).all() and (db == 0).all()
    assert getattr(L, "chela_selscan_bwd" + sfx)(*scan, p(S), x, D, p(S), None, p(dX), p(dZ), p(dA), p(dB), p(dC), None, None, None, p(S2), st) == 0
    assert (dA == 0).all()
    for in_place in (False, True):
        assert getattr(L, "chela_short_conv_fwd" + sfx)(*conv, p(C), p(C if in_place else C2), None, 0, p(dX), st) == 0
        assert getattr(L, "chela_selscan_fwd" + sfx)(*scan, p(S), p(S if in_place else S2), None, 0, p(dX), None, st) == 0
    assert (dX == 3).all() and (dZ == 3).all() and (dB == 3).all() and (dC == 3).all()
    assert all((t == 5).all() for t in (S, S2, C, C2))


def test_what_is_not_finite_stays_in_its_sequence():
    r, D, N, m = gen(19), 64, 16, 4
    lens = [20, 30, 25]
    T, o = sum(lens), offsets(lens)
    u, delta, z, Bm, Cm, A, skip, bias = scan_inputs(r, T, D, N, 1, F32)
    dY, w, cu = r(T, D), r(D, m), cu_of(lens)
    kw = dict(D=skip, Z=z, delta_bias=bias, cu=cu)
    clean = binding.chela_selscan_fwd(u, delta, A, Bm, Cm, **kw)[0]
    g0 = binding.chela_selscan_bwd(u, delta, A, Bm, Cm, dY, **kw)
    c0, h0 = binding.chela_short_conv_fwd(u, w, cu=cu), binding.chela_short_conv_bwd(u, w, dY, cu=cu)
    for value in (float("nan"), float("inf")):
        v = u.clone()
        v[o[1] + 7, 5] = value
        Y = binding.chela_selscan_fwd(v, delta, A, Bm, Cm, **kw)[0]
        g = binding.chela_selscan_bwd(v, delta, A, Bm, Cm, dY, **kw)
        c, h = binding.chela_short_conv_fwd(v, w, cu=cu), binding.chela_short_conv_bwd(v, w, dY, cu=cu)
        keep = torch.ones(T, dtype=torch.bool, device="cuda")
        keep[o[1]:o[2]] = False
        assert not torch.isfinite(Y[o[1] + 7, 5]) and not torch.isfinite(c[o[1] + 7, 5])
        assert torch.equal(Y[keep], clean[keep]) and torch.equal(c[keep], c0[keep]) and torch.equal(h[0][keep], h0[0][keep])
        for k in (0, 1, 3, 4, 6):
            assert torch.equal(g[k][keep], g0[k][keep]), k
        assert torch.equal(Y[o[1]:o[1] + 7], clean[o[1]:o[1] + 7])          # causal
        others = [i for i in range(D) if i != 5]
        assert torch.equal(Y[:, others], clean[:, others])                  # channel by channel


def test_selscan_extreme_steps_and_decays():
    # step sizes that end a state at once, that change nothing, growing states; all against the definition
    r, D, N, L = gen(23), 64, 8, 60
    u, delta, z, Bm, Cm, A, skip, bias = scan_inputs(r, L, D, N, 1, F32)
    delta[::7] = 60.0
    delta[3::7] = -60.0
    A[0], A[1] = 0.0, 0.01
    Y, _ = binding.chela_selscan_fwd(u, delta, A, Bm, Cm, Z=z)
    dY = r(L, D)
    g = binding.chela_selscan_bwd(u, delta, A, Bm, Cm, dY, Z=z)
    n64 = [f64(t) for t in (u, delta, A, Bm, Cm)]
    f, mf = R.selscan_fwd(*n64, None, f64(z))
    v, mv = R.selscan_bwd(*n64, f64(dY), None, f64(z))
    # (an exponent of up to 60 * e^3: its rounding costs as many steps)
    k = 8 * L + 128 + 3000
    check("Y", Y, f["Y"], mf["Y"], k)
    for i, name in enumerate(("dU", "ddelta", "dA", "dB", "dC")):
        check(name, g[i], v[name], mv[name], 2 * k)


def test_selscan_growth_over_rows_that_bring_nothing():
    # states of zero under a growth that no float holds over a chunk of rows, in front of the first input and behind the last gradient
    r, D, N, L = gen(59), 64, 8, 600
    u, delta, z, Bm, Cm, A, skip, bias = scan_inputs(r, L, D, N, 1, F32)
    A = torch.linspace(0.25, 2.0, N, device="cuda")[:, None].expand(N, D).contiguous()
    u[:590] = 0
    delta[:] = 0.5413                                                   # steps of 1: up to e^2 a row, e^96 over 48 rows
    Y, _ = binding.chela_selscan_fwd(u, delta, A, Bm, Cm)
    f, mf = R.selscan_fwd(*[f64(t) for t in (u, delta, A, Bm, Cm)])
    assert (Y[:590] == 0).all()
    check("Y", Y, f["Y"], mf["Y"], 8 * 10 + 128)
    u, dY = r(L, D), r(L, D)
    dY[10:] = 0
    g = binding.chela_selscan_bwd(u[:40], delta[:40], A, Bm[:40], Cm[:40], dY[:40])
    far = binding.chela_selscan_bwd(u, delta, A, Bm, Cm, dY)
    for k in (0, 3):                                                    # (what reaches back from the first ten rows)
        assert torch.equal(far[k][:10], g[k][:10]) and (far[k][10:] == 0).all(), k


@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("T,first,D,N", [(2400, 768, 64, 8), (2400, 700, 64, 16), (700, 24, 64, 32), (3000, 0, 2100, 8)])
def test_selscan_states_that_last_where_no_decay_does(T, first, D, N, sign):
    # over 700 rows that bring nothing a state grows from 1e-12 by 2^140, or shrinks from 1e30 by as much: each row's state is a
    # float, what the chunks' decays make together is none.  The same for the gradient on its way back.
    r, rows = gen(97 + T + N), min(700, T - first)
    A = torch.full((N, D), sign * 0.5, device="cuda")
    delta = torch.zeros(T, D, device="cuda")
    delta[first:first + rows] = 140 / rows / (0.5 * 1.4426950408889634)
    u, dY = torch.zeros(T, D, device="cuda"), torch.zeros(T, D, device="cuda")
    Bm, Cm = r(T, 1, N), r(T, 1, N)
    S = (1e-12 if sign > 0 else 1e30) * (1 + r(1, N, D).abs())
    kw = dict(softplus=False, S_in=S)
    S_out = torch.empty_like(S)
    Y, _ = binding.chela_selscan_fwd(u[None], delta[None], A, Bm[None], Cm[None], S_out=S_out, **kw)
    n64 = [f64(t) for t in (u, delta, A, Bm, Cm)]
    f, mf = R.selscan_fwd(*n64, softplus=False, state=f64(S)[0])
    # (an exponent of 97, made of sums of 24 and of 32 step sizes: 97 * 60 roundings, fewer than these)
    n = 8 * T + 128
    check("Y", Y[0], f["Y"], mf["Y"], n)
    check("S_out", S_out[0], f["S_out"], mf["S_out"], n)
    g = binding.chela_selscan_bwd(u[None], delta[None], A, Bm[None], Cm[None], dY[None], softplus=False, dS_out=S, want_dS_in=True)
    v, mv = R.selscan_bwd(*n64, f64(dY), softplus=False, dstate=f64(S)[0])
    for name, t in (("dU", g[0][0]), ("ddelta", g[1][0]), ("dA", g[2]), ("dS_in", g[8][0])):
        check(name, t, v[name], mv[name], 2 * n)


# ------------------------------------------------------------------------------------------- norms around a block
NORM = [  # rows, D, gate, w_post, w_pre, Y, fp32 stream
    (1, 64, True, True, True, True, False),
    (5, 768, True, True, True, True, False),
    (9, 768, True, True, True, True, True),
    (4, 1, True, True, True, True, False),
    (7, 33, True, False, True, True, False),
    (3, 512, False, True, True, True, True),
    (6, 1000, True, True, False, True, False),
    (3, 1531, True, True, True, True, False),
    (2, 2048, False, False, True, True, False),
    (3, 2056, True, True, True, True, False),
    (2, 4096, True, True, True, True, False),
    (2, 8192, True, True, True, True, True),
    (3, 5001, True, True, True, True, False),
    (1030, 200, True, True, True, True, False),
    (2100, 1100, True, True, True, True, False),
    (6, 768, False, False, True, False, False),
    (2, 300, False, False, True, False, True),
    (5, 2, True, True, True, True, False),
    (6, 3, True, True, True, True, True),
    (3, 4095, True, True, True, True, True),
    (2, 8190, True, True, True, True, False),
    (2, 8191, True, True, True, True, True),
]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,D,gated,post,pre,block,x_f32", NORM)
def test_block_norm(dtype, rows, D, gated, post, pre, block, x_f32):
    r = gen(rows + D)
    xt = F32 if x_f32 and block else dtype
    Y = r(rows, D).to(dtype) if block else None
    X, gate = (2 * r(rows, D)).to(xt), r(rows, D).to(dtype) if gated else None
    wp, wn = (1 + 0.3 * r(D) if on else None for on in (post, pre))
    kw = dict(gate=gate, w_post=wp, w_pre=wn, scale=0.7, eps=1e-5)
    X_out, Nrm = binding.chela_block_norm_fwd(Y, X, **kw)
    n64 = {k: f64(v) if isinstance(v, torch.Tensor) else v for k, v in kw.items()}
    f, mf = R.block_norm_fwd(f64(Y) if block else None, f64(X), **n64)
    if block:
        check("X_out", X_out, f["X_out"], mf["X_out"], D + 64)
        X2 = X.clone()
        a, b = binding.chela_block_norm_fwd(Y, X2, X_out=X2, **kw)
        assert torch.equal(a, X_out) and (Nrm is None or torch.equal(b, Nrm))
    else:
        assert X_out is X
    if pre:
        check("N", Nrm, f["N"], mf["N"], D + 64)
    else:
        assert Nrm is None
    for upstream in (True, False):
        dX_out = r(rows, D).to(xt) if upstream else None
        if not upstream and not pre:
            continue
        dN = r(rows, D).to(dtype) if pre else None
        g = binding.chela_block_norm_bwd(Y, X_out, dX_out, dN, **kw)
        v, mv = R.block_norm_bwd(f64(Y) if block else None, f64(X_out), None if dX_out is None else f64(dX_out), None if dN is None else f64(dN), **n64)
        for name, t in zip(("dY", "dgate", "dX", "dw_post", "dw_pre"), g):
            assert (t is None) == (name not in v), name
            if t is not None:
                check(name, t, v[name], mv[name], 2 * (D + 64) + (rows if name.startswith("dw") else 0))
        if upstream:
            again = binding.chela_block_norm_bwd(Y, X_out, dX_out, dN, in_place=True, **kw)
            assert again[2] is dX_out
            assert all([same(a, b) for a, b in zip(g, again)])


@pytest.mark.parametrize("D", [768, 1531, 4506])
@pytest.mark.parametrize("dtype", DTYPES)
def test_block_norm_in_place_of_a_tensor_that_is_there_twice(dtype, D):
    # one tensor as both upstream gradients, or as the block's output and the stream: a thread reads of it what it writes
    r, n = gen(D), 300
    Y, X, gate, d, wp, wn = r(n, D).to(dtype), r(n, D).to(dtype), r(n, D).to(dtype), r(n, D).to(dtype), 1 + 0.1 * r(D), 1 + 0.1 * r(D)
    kw = dict(gate=gate, w_post=wp, w_pre=wn, scale=0.5)
    want = binding.chela_block_norm_bwd(Y, X, d, d, **kw)
    d2 = d.clone()
    got = binding.chela_block_norm_bwd(Y, X, d2, d2, in_place=True, **kw)
    assert got[2] is d2 and all([torch.equal(a, b) for a, b in zip(want, got)])
    want = binding.chela_block_norm_fwd(X, X, **kw)
    X2 = X.clone()
    got = binding.chela_block_norm_fwd(X2, X2, X_out=X2, **kw)
    assert got[0] is X2 and all([torch.equal(a, b) for a, b in zip(want, got)])
    if dtype == BF:                                                      # rows of another size at one address: refused
        whole = torch.zeros(n, D, device="cuda")
        with pytest.raises(binding.ChelaError) as e:
            binding.chela_block_norm_fwd(whole.view(-1).view(BF)[:n * D].view(n, D), whole, X_out=whole, w_pre=wn)
        assert e.value.status == -6


def test_block_norm_of_zeros():
    x = torch.zeros(3, 64, device="cuda")
    w = torch.ones(64, device="cuda")
    assert (binding.chela_block_norm_fwd(None, x, w_pre=w)[1] == 0).all()
    assert torch.isnan(binding.chela_block_norm_fwd(None, x, w_pre=w, eps=0.0)[1]).all()           # as the formula says
    x[1, 3] = float("inf")
    n = binding.chela_block_norm_fwd(None, x, w_pre=w)[1]
    assert (n[0] == 0).all() and (n[2] == 0).all() and torch.isnan(n[1, 3])


# ------------------------------------------------------------------------------------------- together
def test_a_block_of_all_three_prompt_then_tokens_is_the_sequence():
    # norm, convolution, scan, norm with gate and residual, over whole sequences and over prompts followed by single tokens
    r, n, L, D, N, m, k = gen(29), 3, 90, 64, 16, 4, 77
    X = r(n, L, D).to(BF)
    w, cb, A, skip, bias = 0.5 * r(D, m), 0.1 * r(D), -torch.exp(r(N, D)), r(D), r(D) - 2
    wp, wn = 1 + 0.1 * r(D), 1 + 0.1 * r(D)
    mix = r(D, D + 2 * N).to(BF) / 8

    def block(x, conv, scan):
        h = binding.chela_block_norm_fwd(None, x, w_pre=wn)[1]
        c = conv(h)
        p = (c.float().reshape(-1, D) @ mix.float()).to(BF).view(*c.shape[:-1], D + 2 * N)     # (row by row the same sums, up to their order)
        y = scan(c, p[..., :D], p[..., D:D + N], p[..., D + N:], h)
        return binding.chela_block_norm_fwd(y, x, gate=h, w_post=wp, w_pre=wn, scale=0.5)

    def whole(x, C, S):
        return block(x, lambda h: binding.chela_short_conv_fwd(h, w, bias=cb, S_in=C, S_out=C),
                     lambda c, d, Bm, Cm, z: binding.chela_selscan_fwd(c, d, A, Bm, Cm, D=skip, Z=z, delta_bias=bias, S_in=S, S_out=S)[0])

    def token(x, C, S):
        return block(x, lambda h: binding.chela_short_conv_step(h, w, C, bias=cb),
                     lambda c, d, Bm, Cm, z: binding.chela_selscan_step(c, d, A, Bm, Cm, S, D=skip, z=z, delta_bias=bias))

    def fresh():
        return torch.zeros(n, m - 1, D, dtype=BF, device="cuda"), torch.zeros(n, N, D, device="cuda")

    C, S = fresh()
    one = whole(X, C, S)
    c2, s2 = fresh()
    parts = [whole(X[:, :k].contiguous(), c2, s2)]
    parts += [tuple(t[:, None] for t in token(X[:, t].contiguous(), c2, s2)) for t in range(k, L)]
    # every stage rounds to bf16, and sums taken in another order may round the other way: a few steps of the largest values
    for i in range(2):
        got = torch.cat([p[i] for p in parts], 1).float()
        assert (got - one[i].float()).abs().max() <= 8 * 2.0 ** -8 * one[i].float().abs().max()
    assert torch.equal(C, c2)
    assert (S - s2).abs().max() <= 8 * 2.0 ** -8 * S.abs().max()


# ------------------------------------------------------------------------------------------- streams, graphs, sizes
def _training_pass(D, N, m, T, dtype, seed):
    r = gen(seed)
    u, delta, z, Bm, Cm, A, skip, bias = scan_inputs(r, T, D, N, 1, dtype)
    w, dY, wp = r(D, m), r(T, D).to(dtype), 1 + 0.1 * r(D)
    cu = cu_of([T // 3, T - T // 3])

    def run():
        kw = dict(D=skip, Z=z, delta_bias=bias, cu=cu)
        c = binding.chela_short_conv_fwd(u, w, cu=cu)
        Y, saved = binding.chela_selscan_fwd(c, delta, A, Bm, Cm, want_saved=True, **kw)
        X, n = binding.chela_block_norm_fwd(Y, u, gate=z, w_post=wp, w_pre=wp)
        b = binding.chela_block_norm_bwd(Y, X, dY, dY, gate=z, w_post=wp, w_pre=wp)
        g = binding.chela_selscan_bwd(c, delta, A, Bm, Cm, b[0], saved=saved, **kw)
        h = binding.chela_short_conv_bwd(u, w, g[0], cu=cu)
        return [t for t in (c, Y, X, n, *b, *g, *h) if t is not None]

    return run, (u, delta, z, dY)


def test_on_another_stream_and_two_at_once():
    run, _ = _training_pass(256, 16, 4, 500, BF, 31)
    run2, _ = _training_pass(192, 8, 3, 700, F32, 37)
    a, b = run(), run2()
    torch.cuda.synchronize()
    s, t = torch.cuda.Stream(), torch.cuda.Stream()
    with torch.cuda.stream(s):
        a1 = run()
    with torch.cuda.stream(t):
        b1 = run2()
    with torch.cuda.stream(s):
        a2 = run()
    torch.cuda.synchronize()
    for x, y in ((a, a1), (a, a2), (b, b1)):
        for p, q in zip(x, y):
            assert torch.equal(p, q)


def test_captured_and_replayed():
    run, inputs = _training_pass(256, 16, 4, 500, BF, 41)
    ws = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")
    s = torch.cuda.Stream()
    binding.chela_set_workspace(ws)
    try:
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            run()
        torch.cuda.current_stream().wait_stream(s)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            out = run()
    finally:
        binding.chela_set_workspace(None)
    other = gen(43)
    for k in range(4):
        for t in inputs:
            t.copy_(other(*t.shape).to(t.dtype))
        want = run()                                       # eagerly, between the replays
        for t in out:
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        for p, q in zip(out, want):
            assert torch.equal(p, q), k


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D", [64, 33])
def test_the_compiled_host_path_and_the_binding_do_the_same(dtype, D):
    # (with a stream named, a call goes through the binding's own lines)
    r, m, N, n, L = gen(61 + D), 4, 8, 3, 50
    here = torch.cuda.current_stream()
    u, delta, z, Bm, Cm, A, skip, bias = scan_inputs(r, n * L, D, N, 1, dtype)
    w, cu = r(D, m), cu_of([20, 0, 100, 25])
    slots, slots4 = torch.tensor([4, 0, -1], dtype=torch.int32, device="cuda"), torch.tensor([1, 3, 2, 0], dtype=torch.int32, device="cuda")
    conv, pool = r(5, m - 1, D).to(dtype), r(5, N, D)
    b3 = lambda t: t.view(n, L, t.shape[-1])  # noqa: E731
    wide = wide_rows(u)

    def both(f, *args, states=(), **kw):
        out = []
        for s in (None, here):
            own = {k: v.clone() for k, v in states}
            kw = {k: v.clone() if k in ("Y", "y") else v for k, v in kw.items()}
            if "S_in" in own:
                own["S_out"] = own["S_in"]
            y = f(*args, stream=s, **own, **kw)
            out.append([t for t in (y if isinstance(y, tuple) else (y,)) if t is not None] + list(own.values()))
        bits = lambda t: t.contiguous().view(torch.int16 if t.dtype == BF else torch.int32)  # noqa: E731  (of what is no number, too)
        for a, b in zip(*out):
            assert a.shape == b.shape and a.dtype == b.dtype
            if "cu" in kw and a.shape[0] == n * L:
                a, b = a[:145], b[:145]                                  # (the others are of no sequence: new tensors hold anything there)
            assert torch.equal(bits(a), bits(b))

    for x, kw in ((u, {}), (b3(u), {}), (wide, {}), (u, dict(cu=cu, silu=False)), (b3(u), dict(bias=bias, Y=torch.empty_like(b3(u))))):
        both(binding.chela_short_conv_fwd, x, w, **kw)
    both(binding.chela_short_conv_fwd, b3(u), w, states=[("S_in", conv)], slots=slots)
    both(binding.chela_short_conv_fwd, u, w, cu=cu, states=[("S_in", conv)], slots=slots4)
    both(binding.chela_short_conv_step, u[:3], w, states=[("S", conv)], slots=slots, bias=bias, y=torch.zeros_like(u[:3]))
    both(binding.chela_short_conv_step, wide[:5], w, states=[("S", conv)], silu=False)
    full = dict(D=skip, delta_bias=bias)
    both(binding.chela_selscan_fwd, u, delta, A, Bm, Cm, cu=cu, **full, Z=z, states=[("S_in", pool)], slots=slots4,
         Y=torch.zeros_like(u))
    both(binding.chela_selscan_fwd, b3(u), b3(delta), A, b3(Bm.flatten(1)), b3(Cm.flatten(1)), want_saved=False, softplus=False)
    both(binding.chela_selscan_fwd, wide, delta, A, Bm, Cm, cu=cu)
    both(binding.chela_selscan_step, u[:3], delta[:3], A, Bm[:3], Cm[:3], states=[("S", pool)], z=z[:3], slots=slots, y=torch.zeros_like(u[:3]), **full)
    both(binding.chela_selscan_step, wide[:5], delta[:5], A, Bm[:5], Cm[:5], states=[("S", pool)])
    g1 = 1 + 0.1 * r(D)
    for kw in (dict(w_pre=g1), dict(gate=z, w_post=g1, w_pre=g1, scale=0.5), dict(w_post=g1)):
        both(binding.chela_block_norm_fwd, u, delta, **kw)
    both(binding.chela_block_norm_fwd, None, b3(u), w_pre=g1)
    dY, dS, dC = r(n * L, D).to(dtype), r(4, N, D), r(4, m - 1, D).to(dtype)
    both(binding.chela_short_conv_bwd, u, w, dY, cu=cu, S_in=conv[:4], dS_out=dC, want_dS_in=True, bias=bias)
    both(binding.chela_short_conv_bwd, b3(u), w, b3(dY), silu=False)
    both(binding.chela_short_conv_bwd, wide, w, wide_rows(dY))
    saved = binding.chela_selscan_fwd(u, delta, A, Bm, Cm, cu=cu, Z=z, S_in=pool[:4], want_saved=True, **full)[1]
    both(binding.chela_selscan_bwd, u, delta, A, Bm, Cm, dY, cu=cu, Z=z, S_in=pool[:4], dS_out=dS, want_dS_in=True, saved=saved, **full)
    both(binding.chela_selscan_bwd, b3(u), b3(delta), A, b3(Bm.flatten(1)), b3(Cm.flatten(1)), b3(dY))
    for kw in (dict(w_pre=g1), dict(gate=z, w_post=g1, w_pre=g1, scale=0.5), dict(w_post=g1)):
        both(binding.chela_block_norm_bwd, u, delta, dY, z if "w_pre" in kw else None, **kw)
    both(binding.chela_block_norm_bwd, u, b3(delta).flatten(0, 1), None, z, w_pre=g1)
    x1, x2 = dY.clone(), dY.clone()
    a = binding.chela_block_norm_bwd(u, delta, x1, z, w_pre=g1, in_place=True)
    b = binding.chela_block_norm_bwd(u, delta, x2, z, w_pre=g1, in_place=True, stream=here)
    assert a[2] is x1 and b[2] is x2 and torch.equal(x1, x2) and not torch.equal(x1, dY) and a[1] is None and a[3] is None
    for bad in (dict(saved=saved[:-4]), dict(saved=saved.double()), dict(dS_out=pool), dict(S_in=dS.double())):
        for s in (None, here):
            with pytest.raises(ValueError):
                binding.chela_selscan_bwd(u, delta, A, Bm, Cm, dY, cu=cu, **dict(dict(stream=s), **bad))
    x1, x2 = u.clone(), u.clone()
    n1, n2 = torch.empty_like(u), torch.empty_like(u)
    a = binding.chela_block_norm_fwd(delta, x1, w_pre=g1, X_out=x1, Nrm=n1)
    b = binding.chela_block_norm_fwd(delta, x2, w_pre=g1, X_out=x2, Nrm=n2, stream=here)
    assert a[0] is x1 and a[1] is n1 and torch.equal(x1, x2) and torch.equal(n1, n2) and not torch.equal(x1, u)
    for bad in (dict(w=w.double()), dict(w=w[1:].contiguous()), dict(bias=bias[1:]), dict(S_in=conv), dict(cu=cu.long()), dict(Y=u[1:])):
        for s in (None, here):
            with pytest.raises(ValueError):
                binding.chela_short_conv_fwd(u, **dict(dict(w=w, stream=s), **bad))


def test_two_graphs_with_the_library_s_own_scratch():
    runs = [_training_pass(256, 16, 4, 500, BF, 67), _training_pass(192, 8, 3, 700, F32, 71)]
    s, graphs, outs = torch.cuda.Stream(), [], []
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        for run, _ in runs:
            run()                                          # (what the stream's scratch has to hold, before anything is captured)
    torch.cuda.current_stream().wait_stream(s)
    for run, _ in runs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            outs.append(run())
        graphs.append(g)
    other = gen(73)
    for k in range(3):
        for _, inputs in runs:
            for t in inputs:
                t.copy_(other(*t.shape).to(t.dtype))
        want = [run() for run, _ in runs]
        for out in outs:
            for t in out:
                t.fill_(float("nan"))
        for g in graphs[::-1] if k % 2 else graphs:
            g.replay()
        torch.cuda.synchronize()
        for out, w in zip(outs, want):
            for p, q in zip(out, w):
                assert torch.equal(p, q), k


def test_two_threads_with_streams_of_their_own():
    import threading
    made = [_training_pass(256, 16, 4, 500, BF, 79), _training_pass(192, 8, 3, 700, F32, 83)]
    want = [run() for run, _ in made]
    torch.cuda.synchronize()
    got, wrong = [None, None], []

    def work(i):
        try:
            s = torch.cuda.Stream()
            with torch.cuda.stream(s):
                for _ in range(5):
                    got[i] = made[i][0]()
            s.synchronize()
        except Exception as e:                             # (a thread's own would be lost)
            wrong.append(e)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong
    for a, b in zip(got, want):
        for p, q in zip(a, b):
            assert torch.equal(p, q)


def test_offsets_beyond_32_bits():
    # the last rows of tensors of more than 2^31 elements
    T, D = 70000, 32768
    w = torch.tensor([[0.5, 0.25]], device="cuda").expand(D, 2).contiguous()
    x = torch.zeros(T, D, dtype=BF, device="cuda")
    r = gen(47)
    x[-40:] = r(40, D).to(BF)
    y = binding.chela_short_conv_fwd(x, w)
    tail, mass, _ = R.short_conv_fwd(f64(x[-41:]), f64(w))
    check("conv", y[-40:], tail[1:], mass[1:], 64)
    assert (y[:-40] == 0).all()
    dX = binding.chela_short_conv_bwd(x, w, x)[0]
    v, mv = R.short_conv_bwd(f64(x[-41:]), f64(w), f64(x[-41:]))
    check("dX", dX[-40:], v["dX"][1:], mv["dX"][1:], 64)
    del dX
    N = 8
    Bm = r(T, N).to(BF)
    A = -torch.ones(N, D, device="cuda")
    y, _ = binding.chela_selscan_fwd(x, x, A, Bm, Bm, Y=y)
    f, mf = R.selscan_fwd(f64(x[-40:]), f64(x[-40:]), f64(A), f64(Bm[-40:])[:, None], f64(Bm[-40:])[:, None])
    check("scan", y[-40:], f["Y"], mf["Y"], 8 * 40 + 128)
    del y
    rows = T * 4
    wn = torch.ones(8192, device="cuda")
    n = binding.chela_block_norm_fwd(None, x.view(rows, 8192), w_pre=wn)[1]
    f, mf = R.block_norm_fwd(None, f64(x.view(rows, 8192)[-5:]), w_pre=f64(wn))
    check("norm", n[-5:], f["N"], mf["N"], 8192 + 64)
