"""Operators on rows without a GPU: the definitions against differences and other forms, the refusals of the library's entry points
and of the binding."""
import numpy as np
import pytest
import torch

from oracle import rows as R


# ------------------------------------------------------------------------------------------- the definitions
def _differences(f, x, h=1e-6):
    """d f / d x by central differences, f a scalar."""
    g = np.zeros(x.shape)
    for i in np.ndindex(x.shape):
        keep = x[i]
        x[i] = keep + h
        up = f()
        x[i] = keep - h
        down = f()
        x[i] = keep
        g[i] = (up - down) / (2 * h)
    return g


def _close(a, b, size=0.0, h=1e-6):
    # central differences: truncation of the order h^2 = 1e-12; and each of the two values whose difference is divided by 2 h has at most 168
    # roundings (8 a row, 128 on top) of its terms' magnitudes, `size`.  (Without softplus half of the step sizes are negative and states
    # grow: at a size of 5e9 a difference of two values, whose last digit alone is 1e-6, says nothing about less than 1.)
    assert np.allclose(a, b, rtol=1e-6, atol=1e-7 + 168 * 2.0 ** -53 * size / h), np.abs(a - b).max()


@pytest.mark.parametrize("act", [True, False])
@pytest.mark.parametrize("L,m", [(1, 4), (2, 4), (7, 4), (5, 1), (6, 2)])
def test_short_conv_gradient_against_differences(rng, act, L, m):
    D = 3
    x, w, b, s = rng.normal(size=(L, D)), rng.normal(size=(D, m)), rng.normal(size=D), rng.normal(size=(m - 1, D))
    dy, ds = rng.normal(size=(L, D)), rng.normal(size=(m - 1, D))

    def loss():
        y, _, after = R.short_conv_fwd(x, w, b, act, s)
        return (y * dy).sum() + (after * ds).sum()

    v, mass = R.short_conv_bwd(x, w, dy, b, act, s, ds)
    for k, t in (("dX", x), ("dw", w), ("dbias", b), ("dS_in", s)):
        _close(v[k], _differences(loss, t))
        assert (np.abs(v[k]) <= mass[k] * (1 + 1e-12) + 1e-15).all()


@pytest.mark.parametrize("softplus,full", [(True, True), (False, True), (True, False)])
@pytest.mark.parametrize("L", [1, 5])
def test_selscan_gradient_against_differences(rng, softplus, full, L):
    D, N, G = 4, 3, 2
    u, delta = rng.normal(size=(L, D)), rng.normal(size=(L, D))
    A, Bm, Cm = -np.exp(rng.normal(size=(N, D))), rng.normal(size=(L, G, N)), rng.normal(size=(L, G, N))
    skip, z, b = (rng.normal(size=D), rng.normal(size=(L, D)), rng.normal(size=D)) if full else (None, None, None)
    s, dY, ds = rng.normal(size=(N, D)), rng.normal(size=(L, D)), rng.normal(size=(N, D))

    def loss():
        v, _ = R.selscan_fwd(u, delta, A, Bm, Cm, skip, z, b, softplus, s)
        return (v["Y"] * dY).sum() + (v["S_out"] * ds).sum()

    f = R.selscan_fwd(u, delta, A, Bm, Cm, skip, z, b, softplus, s)[1]
    size = (f["Y"] * np.abs(dY)).sum() + (f["S_out"] * np.abs(ds)).sum()
    v, mass = R.selscan_bwd(u, delta, A, Bm, Cm, dY, skip, z, b, softplus, s, ds)
    for k, t in (("dU", u), ("ddelta", delta), ("dA", A), ("dB", Bm), ("dC", Cm), ("dD", skip), ("dZ", z), ("dbias", b), ("dS_in", s)):
        if t is None:
            continue
        _close(v[k], _differences(loss, t), size)
        assert (np.abs(v[k]) <= mass[k] * (1 + 1e-12) + 1e-15).all(), k


@pytest.mark.parametrize("gated,post,pre", [(True, True, True), (False, True, True), (True, False, True), (True, True, False), (False, False, True)])
def test_block_norm_gradient_against_differences(rng, gated, post, pre):
    n, D, scale = 3, 5, 0.7
    Y, X = rng.normal(size=(n, D)), rng.normal(size=(n, D))
    gate = rng.normal(size=(n, D)) if gated else None
    wp, wn = (rng.normal(size=D) if on else None for on in (post, pre))
    dX, dN = rng.normal(size=(n, D)), rng.normal(size=(n, D)) if pre else None

    def loss():
        v, _ = R.block_norm_fwd(Y, X, gate, wp, wn, scale)
        return (v["X_out"] * dX).sum() + ((v["N"] * dN).sum() if pre else 0)

    after = R.block_norm_fwd(Y, X, gate, wp, wn, scale)[0]["X_out"]
    v, mass = R.block_norm_bwd(Y, after, dX, dN, gate, wp, wn, scale)
    for k, t in (("dY", Y), ("dgate", gate), ("dX", X), ("dw_post", wp), ("dw_pre", wn)):
        if t is None:
            continue
        _close(v[k], _differences(loss, t))
        assert (np.abs(v[k]) <= mass[k] * (1 + 1e-12) + 1e-15).all(), k


def test_definitions_in_pieces(rng):
    # a sequence in two pieces, the state handed over, and token by token, is the sequence
    L, D, m, N = 9, 4, 4, 3
    x, w = rng.normal(size=(L, D)), rng.normal(size=(D, m))
    whole, _, last = R.short_conv_fwd(x, w)
    s, got = None, []
    for a, b in ((0, 2), (2, 3), (3, 9)):
        y, _, s = R.short_conv_fwd(x[a:b], w, state=s)
        got.append(y)
    assert np.allclose(np.concatenate(got), whole) and np.allclose(s, last) and np.allclose(last, x[-3:])
    delta, A = rng.normal(size=(L, D)), -np.exp(rng.normal(size=(N, D)))
    Bm, Cm = rng.normal(size=(L, 1, N)), rng.normal(size=(L, 1, N))
    whole = R.selscan_fwd(x, delta, A, Bm, Cm)[0]
    s, got = None, []
    for t in range(L):
        v = R.selscan_fwd(x[t:t + 1], delta[t:t + 1], A, Bm[t:t + 1], Cm[t:t + 1], state=s)[0]
        s = v["S_out"]
        got.append(v["Y"])
    assert np.allclose(np.concatenate(got), whole["Y"]) and np.allclose(s, whole["S_out"])


def test_selscan_without_decay_is_a_causal_sum(rng):
    # A = 0 and step sizes of one: the state adds up the rows' products, as the causal linear attention's does
    L, D, N = 12, 2, 3
    u, Bm, Cm = rng.normal(size=(L, D)), rng.normal(size=(L, 1, N)), rng.normal(size=(L, 1, N))
    v = R.selscan_fwd(u, np.ones((L, D)), np.zeros((N, D)), Bm, Cm, softplus=False)[0]
    P = np.tril(Cm[:, 0] @ Bm[:, 0].T)
    assert np.allclose(v["Y"], P @ u) and np.allclose(v["S_out"], Bm[:, 0].T @ u)


@pytest.mark.parametrize("lasting", [False, True])
def test_the_scan_s_bound_tells_a_carry_of_fewer_bits(rng, lasting):
    # a scan in fp32 by chunks of 24 rows: with what the chunks hand on in fp32 it is within the bound, in 16 bits of it it is not
    L, D, N, chunk = 1200, 8, 8, 24
    f4 = np.float32
    u, delta, C, B = (rng.normal(size=s).astype(f4) for s in ((L, D), (L, D), (L, 1, N), (L, 1, N)))
    A = (-np.exp(rng.normal(size=(N, D))) / (64 if lasting else 1)).astype(f4)
    bias, S = (rng.normal(size=D) - 4).astype(f4), rng.normal(size=(N, D)).astype(f4)
    dl = np.logaddexp(0, (delta + bias).astype(np.float64)).astype(f4)
    b = (dl * u)[:, None] * B.transpose(0, 2, 1)

    def walk(h, rows, out=None):
        for t in rows:
            h = np.exp(dl[t] * A) * h + b[t]
            if out is not None:
                out[t] = (C[t, 0][:, None] * h).sum(0)
        return h

    def scan(keep):
        Y, h = np.zeros((L, D), f4), S
        for t in range(0, L, chunk):
            rows = range(t, min(t + chunk, L))
            walk(h, rows, Y)
            decay = np.exp(A * dl[rows.start:rows.stop].sum(0, dtype=f4))
            h = keep(decay * h + walk(np.zeros((N, D), f4), rows))
            assert h.dtype == f4
        return Y

    x = [t.astype(np.float64) for t in (u, delta, A, B, C)]
    ref = R.selscan_fwd(*x, delta_bias=bias.astype(np.float64), state=S.astype(np.float64))[0]["Y"]
    k = R.selscan_roundings(*x, np.ones((L, D)), delta_bias=bias.astype(np.float64), state=S.astype(np.float64))["Y"]
    worst = lambda Y: float((np.abs(Y - ref) / R.tolerance(ref, k, 1, 2.0 ** -24)).max())  # noqa: E731
    assert worst(scan(lambda h: h)) <= 1
    assert worst(scan(lambda h: h.astype(np.float16).astype(f4))) > 2
    assert worst(scan(lambda h: torch.from_numpy(h).bfloat16().float().numpy())) > 10


# ------------------------------------------------------------------------------------------- refusals
A0, SZ = 0x10000, 1 << 40      # made-up aligned addresses far apart: every call below has to be refused (or be empty) before they are used
NULL, SHAPE, DIM, ALIGN, ALIAS, WS = -1, -2, -3, -5, -6, -7


def at(k):
    return A0 + k * SZ


@pytest.fixture(scope="module")
def L():
    from paper_2406_08128_amd import binding
    return binding.lib()


def _conv_fwd(L, sfx="", X=at(0), ldx=64, w=at(1), m=4, bias=at(2), cu=None, n_seq=2, T=8, D=64, S_in=at(3), S_out=at(4), slots=None,
              n_slots=2, Y=at(5)):
    return getattr(L, "chela_short_conv_fwd" + sfx)(X, ldx, w, m, bias, 1, cu, n_seq, T, D, S_in, S_out, slots, n_slots, Y, None)


@pytest.mark.parametrize("sfx", ["", "_f32"])
def test_short_conv_refusals(L, sfx):
    f = lambda **kw: _conv_fwd(L, sfx, **kw)  # noqa: E731
    assert f(X=None) == NULL and f(w=None) == NULL and f(Y=None) == NULL
    assert f(m=0) == SHAPE and f(m=9) == SHAPE and f(T=-1) == SHAPE and f(n_seq=-1) == SHAPE and f(D=-1) == SHAPE and f(D=(1 << 20) + 1) == SHAPE
    assert f(T=7) == SHAPE                                    # not two sequences of one length
    assert f(n_seq=0, n_slots=0) == SHAPE                     # rows of no sequence
    assert f(n_slots=3) == SHAPE                              # three states for two sequences, and no map
    assert f(ldx=63) == SHAPE and f(ldx=1 << 40) == SHAPE
    assert f(T=2 ** 31 - 2) == SHAPE and f(T=2 ** 30, D=2 ** 20, ldx=2 ** 20) == SHAPE
    # threads of a launch stay below 2^32: rows, sequences, requests times 64 channels of them
    assert f(T=2 ** 28) == SHAPE and f(T=2 ** 24, D=1024, ldx=1024) == SHAPE and f(n_seq=2 ** 23, T=2 ** 23, n_slots=2 ** 23) == SHAPE
    assert f(n_seq=2 ** 20, T=2 ** 20, D=512, ldx=512, n_slots=2 ** 20) == SHAPE
    assert f(X=at(0) + 1) == ALIGN and f(Y=at(5) + 8) == ALIGN and f(w=at(1) + 4) == ALIGN and f(S_in=at(3) + 2) == ALIGN
    assert f(cu=at(6) + 2) == ALIGN and f(slots=at(6) + 1) == ALIGN
    assert f(Y=at(0)) == ALIAS and f(Y=at(3)) == ALIAS and f(S_out=at(5)) == ALIAS and f(S_out=at(3) + 16) == ALIAS and f(Y=at(1)) == ALIAS
    assert f(D=0, ldx=0) == 0 and f(T=0, n_seq=0, n_slots=0, X=None, Y=None) == 0
    b = getattr(L, "chela_short_conv_bwd" + sfx)

    def bwd(X=at(0), ldx=64, w=at(1), m=4, bias=at(2), cu=None, n_seq=2, T=8, D=64, S_in=at(3), dY=at(4), lddy=64, dS_out=at(5), dX=at(6),
            dw=at(7), dbias=at(8), dS_in=at(9)):
        return b(X, ldx, w, m, bias, 1, cu, n_seq, T, D, S_in, dY, lddy, dS_out, dX, dw, dbias, dS_in, None)

    assert bwd(dY=None) == NULL and bwd(dX=None) == NULL and bwd(dw=None) == NULL and bwd(dbias=None) == NULL
    assert bwd(m=9) == SHAPE and bwd(lddy=3) == SHAPE and bwd(T=9) == SHAPE
    assert bwd(dX=at(6) + 4) == ALIGN and bwd(dY=at(4) + 1) == ALIGN
    assert bwd(dX=at(4)) == ALIAS and bwd(dS_in=at(5)) == ALIAS and bwd(dw=at(8)) == ALIAS
    s = getattr(L, "chela_short_conv_step" + sfx)

    def step(x=at(0), ldx=64, w=at(1), m=4, S=at(2), slots=None, n_slots=3, R=3, D=64, y=at(3)):
        return s(x, ldx, w, m, None, 1, S, slots, n_slots, R, D, y, None)

    assert step(x=None) == NULL and step(S=None) == NULL and step(y=None) == NULL
    assert step(m=0) == SHAPE and step(R=-1) == SHAPE and step(R=1 << 24, n_slots=1 << 24) == SHAPE and step(n_slots=4) == SHAPE and step(ldx=1) == SHAPE
    assert step(y=at(0)) == ALIAS and step(y=at(2)) == ALIAS and step(S=at(0)) == ALIAS and step(S=at(2) + 8) == ALIGN
    assert step(R=0, n_slots=0, x=None, S=None, y=None) == 0


@pytest.mark.parametrize("sfx", ["", "_f32"])
def test_selscan_refusals(L, sfx):
    f = getattr(L, "chela_selscan_fwd" + sfx)

    def fwd(U=at(0), ldu=64, delta=at(1), ldd=64, A=at(2), Bm=at(3), ldb=32, Cm=at(4), ldc=32, skip=at(5), Z=at(6), ldz=64, bias=at(7), cu=None,
            n_seq=2, T=8, D=64, N=16, G=2, S_in=at(8), S_out=at(9), slots=None, n_slots=2, Y=at(10), saved=at(11)):
        return f(U, ldu, delta, ldd, A, Bm, ldb, Cm, ldc, skip, Z, ldz, bias, 1, cu, n_seq, T, D, N, G, S_in, S_out, slots, n_slots, Y, saved, None)

    assert fwd(U=None) == NULL and fwd(delta=None) == NULL and fwd(A=None) == NULL and fwd(Bm=None) == NULL and fwd(Cm=None) == NULL
    assert fwd(Y=None) == NULL
    assert fwd(N=12) == DIM and fwd(N=64) == DIM and fwd(N=0) == DIM
    assert fwd(G=0) == SHAPE and fwd(G=3) == SHAPE and fwd(T=9) == SHAPE and fwd(T=-8) == SHAPE and fwd(n_slots=1) == SHAPE
    assert fwd(ldu=63) == SHAPE and fwd(ldb=31) == SHAPE and fwd(ldz=1) == SHAPE and fwd(T=2 ** 31 - 8) == SHAPE
    assert fwd(U=at(0) + 1) == ALIGN and fwd(A=at(2) + 4) == ALIGN and fwd(Y=at(10) + 2) == ALIGN and fwd(S_in=at(8) + 4) == ALIGN
    assert fwd(saved=at(11) + 4) == ALIGN
    assert fwd(Y=at(0)) == ALIAS and fwd(Y=at(6)) == ALIAS and fwd(saved=at(10)) == ALIAS and fwd(S_out=at(8) + 64) == ALIAS and fwd(S_out=at(10)) == ALIAS
    assert fwd(T=0, n_seq=0, n_slots=0, U=None, delta=None, Bm=None, Cm=None, Z=None, Y=None) == 0
    b = getattr(L, "chela_selscan_bwd" + sfx)

    def bwd(U=at(0), A=at(2), skip=at(5), Z=at(6), bias=at(7), T=8, D=64, N=16, G=2, S_in=at(8), dY=at(9), lddy=64, dS_out=at(10), saved=at(11),
            dU=at(12), dd=at(13), dA=at(14), dB=at(15), dC=at(16), dD=at(17), dZ=at(18), db=at(19), dS_in=at(20)):
        return b(U, 64, at(1), 64, A, at(3), 32, at(4), 32, skip, Z, 64, bias, 1, None, 2, T, D, N, G, S_in, dY, lddy, dS_out, saved, dU, dd, dA,
                 dB, dC, dD, dZ, db, dS_in, None)

    for k in ("U", "A", "dY", "dU", "dd", "dA", "dB", "dC", "dD", "dZ", "db"):
        assert bwd(**{k: None}) == NULL, k
    assert bwd(N=24) == DIM and bwd(G=5) == SHAPE and bwd(T=3) == SHAPE and bwd(lddy=2) == SHAPE
    assert bwd(dU=at(12) + 2) == ALIGN and bwd(dA=at(14) + 4) == ALIGN and bwd(dS_in=at(20) + 8) == ALIGN
    assert bwd(dU=at(9)) == ALIAS and bwd(dB=at(16)) == ALIAS and bwd(dS_in=at(10)) == ALIAS and bwd(dA=at(2)) == ALIAS
    s = getattr(L, "chela_selscan_step" + sfx)

    def step(u=at(0), ldu=64, A=at(2), N=16, G=2, S=at(5), slots=None, n_slots=3, R=3, D=64, y=at(6)):
        return s(u, ldu, at(1), 64, A, at(3), 32, at(4), 32, None, None, 0, None, 1, S, slots, n_slots, R, D, N, G, y, None)

    assert step(u=None) == NULL and step(S=None) == NULL and step(y=None) == NULL
    assert step(N=20) == DIM and step(G=7) == SHAPE and step(R=-1) == SHAPE and step(n_slots=2) == SHAPE and step(ldu=8) == SHAPE
    assert step(y=at(5)) == ALIAS and step(S=at(2)) == ALIAS and step(S=at(5) + 4) == ALIGN
    assert step(R=0, n_slots=0, u=None) == 0


@pytest.mark.parametrize("sfx", ["", "_f32"])
def test_block_norm_refusals(L, sfx):
    f = getattr(L, "chela_block_norm_fwd" + sfx)

    def fwd(Y=at(0), gate=at(1), X=at(2), w_post=at(3), w_pre=at(4), X_out=at(5), N=at(6), scale=1.0, eps=1e-5, rows=4, D=64, x_f32=0):
        return f(Y, gate, X, w_post, w_pre, X_out, N, scale, eps, rows, D, x_f32, None)

    assert fwd(X=None) == NULL and fwd(X_out=None) == NULL and fwd(N=None) == NULL and fwd(Y=None, w_pre=None) == NULL
    assert fwd(rows=-1) == SHAPE and fwd(D=0) == SHAPE and fwd(D=8193) == DIM and fwd(rows=1 << 31) == SHAPE
    for bad in (float("nan"), float("inf"), -1.0):
        assert fwd(eps=bad) == SHAPE
    assert fwd(scale=float("nan")) == SHAPE and fwd(scale=float("inf")) == SHAPE
    assert fwd(X=at(2) + 8) == ALIGN and fwd(w_pre=at(4) + 4) == ALIGN
    assert fwd(X_out=at(0)) == ALIAS and fwd(N=at(2)) == ALIAS and fwd(N=at(5)) == ALIAS and fwd(X_out=at(2) + 16) == ALIAS
    assert fwd(rows=0, Y=None, X=None, X_out=None, N=None) == 0
    b = getattr(L, "chela_block_norm_bwd" + sfx)

    def bwd(Y=at(0), gate=at(1), X=at(2), w_post=at(3), w_pre=at(4), dX_out=at(5), dN=at(6), dY=at(7), dgate=at(8), dX=at(9), dwp=at(10), dwn=at(11),
            scale=1.0, eps=1e-5, rows=4, D=64):
        return b(Y, gate, X, w_post, w_pre, dX_out, dN, dY, dgate, dX, dwp, dwn, scale, eps, rows, D, 0, None)

    for k in ("X", "dN", "dY", "dgate", "dX", "dwp", "dwn"):
        assert bwd(**{k: None}) == NULL, k
    assert bwd(D=9000) == DIM and bwd(rows=-3) == SHAPE and bwd(eps=-1.0) == SHAPE
    assert bwd(dX=at(9) + 2) == ALIGN and bwd(dX=at(2)) == ALIAS and bwd(dY=at(8)) == ALIAS and bwd(dX=at(5) + 16) == ALIAS


@pytest.mark.parametrize("sfx", ["", "_f32"])
def test_the_calls_that_clear_refuse_the_same(L, sfx):
    f, b, s = (getattr(L, "chela_short_conv_%s_cleared%s" % (k, sfx)) for k in ("fwd", "bwd", "step"))
    conv = (at(0), 64, at(1), 4, None, 1)
    assert f(*conv, None, 2, 8, 64, None, None, None, 2, None, None) == NULL and f(*conv, None, 2, 8, 64, None, None, None, 2, at(0), None) == ALIAS
    assert b(*conv, None, 2, 9, 64, None, at(2), 64, None, at(3), at(4), None, None, None) == SHAPE
    assert b(*conv, None, 2, 8, 64, None, at(2), 64, None, at(2), at(4), None, None, None) == ALIAS
    assert s(*conv, at(2), None, 3, 3, 64, at(3) + 4, None) == ALIGN and s(*conv, at(2), None, 3, 2, 64, at(3), None) == SHAPE
    f, b, s = (getattr(L, "chela_selscan_%s_cleared%s" % (k, sfx)) for k in ("fwd", "bwd", "step"))
    scan = (at(0), 64, at(1), 64, at(2), at(3), 16, at(4), 16, None, None, 0, None, 1)
    assert f(*scan, None, 2, 8, 64, 12, 1, None, None, None, 2, at(5), None, None) == DIM
    assert f(*scan, None, 2, 8, 64, 16, 1, None, None, None, 2, None, None, None) == NULL
    outs = (at(6), at(7), at(8), at(9), at(10), None, None, None, None, None)
    assert b(*scan, None, 2, 7, 64, 16, 1, None, at(5), 64, None, None, *outs) == SHAPE
    assert b(*scan, None, 2, 8, 64, 16, 1, None, at(6), 64, None, None, *outs) == ALIAS
    assert s(*scan, at(5), None, 3, 3, 64, 16, 1, at(5), None) == ALIAS and s(*scan, at(5), None, 3, 3, 64, 16, 1, None, None) == NULL


@pytest.mark.parametrize("sfx", ["", "_f32"])
def test_only_the_named_input_may_be_where_an_output_is(L, sfx):
    # in place, and another input at the same address: other workgroups read it after one has written
    S, X, w = at(0), at(1), at(2)
    f = getattr(L, "chela_short_conv_fwd" + sfx)
    for kw in (dict(w=S), dict(bias=S), dict(cu=S), dict(slots=S), dict(X=S)):
        a = dict(dict(X=X, w=w, bias=None, cu=None, slots=None), **kw)
        assert f(a["X"], 64, a["w"], 4, a["bias"], 1, a["cu"], 2, 8, 64, S, S, a["slots"], 2, at(3), None) == ALIAS, kw
    f = getattr(L, "chela_selscan_fwd" + sfx)
    names = ("U", "delta", "A", "Bm", "Cm", "skip", "Z", "bias", "cu", "slots")
    for k in names:
        a = dict({n: at(4 + i) for i, n in enumerate(names)}, cu=None, slots=None)
        a[k] = S
        assert f(a["U"], 64, a["delta"], 64, a["A"], a["Bm"], 16, a["Cm"], 16, a["skip"], a["Z"], 64, a["bias"], 1, a["cu"], 1, 8, 64, 16, 1, S, S,
                 a["slots"], 1, at(3), None, None) == ALIAS, k
    f, b = getattr(L, "chela_block_norm_fwd" + sfx), getattr(L, "chela_block_norm_bwd" + sfx)
    for x_f32 in (0, 1):
        for k in range(5):
            a = [at(4), at(5), S, at(6), at(7)]              # Y, gate, X, w_post, w_pre
            if k == 2 or (k < 2 and not (x_f32 and sfx == "")):
                continue                                     # (rows of the stream's type, element by element where the stream's are)
            a[k] = S
            assert f(*a, S, at(8), 1.0, 1e-5, 4, 64, x_f32, None) == ALIAS, k
            a[2] = X
            assert b(*a, S, at(9), at(10), at(11), S, at(12), at(13), 1.0, 1e-5, 4, 64, x_f32, None) == ALIAS, k
    if sfx == "":
        assert b(at(4), at(5), X, at(6), at(7), S, S, at(10), at(11), S, at(12), at(13), 1.0, 1e-5, 4, 64, 1, None) == ALIAS
    assert b(at(4), at(5), S, at(6), at(7), at(8), at(9), at(10), at(11), S, at(12), at(13), 1.0, 1e-5, 4, 64, 0, None) == ALIAS
    assert b(at(4), at(5), S, at(6), at(7), None, at(9), at(10), at(11), S, at(12), at(13), 1.0, 1e-5, 4, 64, 0, None) == ALIAS


def test_workspace_and_saved_queries(L):
    assert L.chela_selscan_saved_bytes(1000, 100, 16) == 125 * 16 * 100 * 4
    assert L.chela_selscan_saved_bytes(0, 100, 16) == 0 and L.chela_selscan_saved_bytes(5, 100, 15) == 0
    for bad in ((0, 64, 16, 1, 0, 0), (8, 0, 16, 1, 0, 0), (8, 64, 12, 1, 0, 0), (8, 64, 16, 0, 0, 0), (8, 64, 16, 3, 1, 0)):
        assert L.chela_selscan_workspace_bytes(*bad) == 0, bad
    a, b = L.chela_selscan_workspace_bytes(4096, 512, 16, 1, 1, 1), L.chela_selscan_workspace_bytes(4096, 512, 16, 1, 1, 0)
    assert 0 < L.chela_selscan_workspace_bytes(4096, 512, 16, 1, 0, 0) < a < b      # the states in front of the tiles come on top
    assert L.chela_selscan_workspace_bytes(2 ** 28, 64, 16, 1, 0, 0) == 0 and L.chela_selscan_saved_bytes(2 ** 24, 1024, 16) == 0
    assert L.chela_short_conv_bwd_workspace_bytes(2 ** 28, 64, 4, 0) == 0
    assert L.chela_short_conv_bwd_workspace_bytes(64, 512, 4, 0) > 0 and L.chela_short_conv_bwd_workspace_bytes(64, 512, 9, 0) == 0
    assert L.chela_block_norm_bwd_workspace_bytes(10, 64) > 0 and L.chela_block_norm_bwd_workspace_bytes(10, 8193) == 0


def test_a_workspace_that_is_too_small_is_refused(L):
    L.chela_set_workspace(A0, 256)
    try:
        f = L.chela_selscan_fwd
        assert f(at(0), 64, at(1), 64, at(2), at(3), 16, at(4), 16, None, None, 0, None, 1, None, 2, 8, 64, 16, 1, None, None, None, 2, at(5), None,
                 None) == WS
        assert L.chela_short_conv_bwd(at(0), 64, at(1), 4, None, 1, None, 2, 8, 64, None, at(2), 64, None, at(3), at(4), None, None, None) == WS
        assert L.chela_block_norm_bwd(None, None, at(0), None, at(1), None, at(2), None, None, at(3), None, at(4), 1.0, 1e-5, 4, 64, 0, None) == WS
    finally:
        L.chela_set_workspace(None, 0)


def test_binding_refuses_what_it_cannot_hand_on():
    from paper_2406_08128_amd import binding
    x, w = torch.zeros(4, 8), torch.zeros(8, 4)
    with pytest.raises(ValueError):
        binding.chela_short_conv_fwd(x, w)                   # not on a device
    with pytest.raises(ValueError):
        binding.chela_selscan_fwd(x, x, torch.zeros(16, 8), torch.zeros(4, 16), torch.zeros(4, 16))
    with pytest.raises(ValueError):
        binding.chela_block_norm_fwd(None, x, w_pre=torch.ones(8))
    with pytest.raises(ValueError):
        binding.chela_short_conv_step(x, w, torch.zeros(4, 3, 8))
    with pytest.raises(ValueError):
        binding.chela_selscan_step(x, x, torch.zeros(16, 8), torch.zeros(4, 16), torch.zeros(4, 16), torch.zeros(4, 16, 8))
    assert binding._row_stride(torch.zeros(4, 20)[:, 3:11], x, "t") [1] == 20
    assert binding._row_stride(torch.zeros(2, 3, 20)[:, :, :8], torch.zeros(2, 3, 8), "t")[1] == 20
    assert binding._row_stride(torch.zeros(4, 40)[:, :32].unflatten(1, (2, 16)), x, "t")[1] == 40
    for bad in (torch.zeros(8, 4).t(), torch.zeros(4, 16)[:, ::2]):
        with pytest.raises(ValueError):
            binding._row_stride(bad, x, "t")
    with pytest.raises(ValueError):
        binding._row_stride(torch.zeros(2, 5, 8)[:, :3], torch.zeros(2, 3, 8), "t")        # rows not evenly spaced
    with pytest.raises(ValueError):
        binding._row_stride(torch.zeros(4, 2, 20)[:, :, :16], x, "t")                       # a row in two pieces
