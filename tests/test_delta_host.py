"""The gated delta rule and the layer norm without a GPU: the definitions against differences, other forms and their bounds, the refusals of
the library's entry points and of the binding."""
import numpy as np
import pytest
import torch

from oracle import delta as R


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


def _inputs(rng, L, dk, dv, weak=2.0):
    def unit(x):
        return x / np.linalg.norm(x, axis=1, keepdims=True)
    return (unit(rng.normal(size=(L, dk))), unit(rng.normal(size=(L, dk))), rng.normal(size=(L, dv)), -np.exp(rng.normal(size=L) - weak),
            1 / (1 + np.exp(-rng.normal(size=L))))


@pytest.mark.parametrize("gated", [True, False])
@pytest.mark.parametrize("L", [1, 6])
def test_delta_gradient_against_differences(rng, L, gated):
    q, k, v, g, beta = _inputs(rng, L, 4, 3)
    g = g if gated else None
    S, dO, dS = rng.normal(size=(4, 3)), rng.normal(size=(L, 3)), rng.normal(size=(4, 3))

    def loss():
        o, s = R.delta_fwd(q, k, v, g, beta, 0.7, S)
        return (o * dO).sum() + (s * dS).sum()

    out = R.delta_bwd(q, k, v, g, beta, dO, 0.7, S, dS)
    for n, t in (("dQ", q), ("dK", k), ("dV", v), ("dg", g), ("dbeta", beta), ("dS_in", S)):
        if t is not None:
            # truncation of the order of h^2, and some hundred roundings of 2^-53 of terms of the order of one over 2 h
            assert np.allclose(out[n], _differences(loss, t), rtol=1e-6, atol=1e-7), n


def test_delta_in_pieces_and_as_corrections(rng):
    q, k, v, g, beta = _inputs(rng, 11, 5, 4)
    whole, last = R.delta_fwd(q, k, v, g, beta)
    S, got = None, []
    for a, b in ((0, 3), (3, 4), (4, 11)):
        o, S = R.delta_fwd(q[a:b], k[a:b], v[a:b], g[a:b], beta[a:b], state=S)
        got.append(o)
    assert np.allclose(np.concatenate(got), whole) and np.allclose(S, last)
    # keys at right angles, nothing decays, beta of one: the state holds every value at its key
    k = np.eye(5)
    o, S = R.delta_fwd(k, k, v[:5], None, np.ones(5))
    assert np.allclose(o, v[:5]) and np.allclose(k @ S, v[:5])
    # and one key for all: the last value
    k = np.tile(np.eye(5)[:1], (5, 1))
    assert np.allclose(R.delta_fwd(k, k, v[:5], None, np.ones(5))[1][0], v[4])


def _chunked(q, k, v, g, beta, C, once, twice):
    """O and S_out by chunks in 32 bits, operands of products rounded by `once` and `twice`."""
    f = np.float32
    q, k, v, g, beta = (x.astype(f) for x in (q, k, v, g, beta))
    S, out = np.zeros((k.shape[1], v.shape[1]), f), []
    for a in range(0, len(k), C):
        K, Q, V, be = k[a:a + C], q[a:a + C], v[a:a + C], beta[a:a + C, None]
        gamma = np.cumsum(g[a:a + C].astype(np.float64))
        D = np.tril(np.exp(np.tril(gamma[:, None] - gamma[None]))).astype(f)
        up, down, whole = np.exp(gamma).astype(f)[:, None], np.exp(gamma[-1] - gamma).astype(f)[:, None], f(np.exp(gamma[-1]))
        T = np.linalg.inv((np.eye(len(K)) + np.tril(be * D * (K @ K.T), -1)).astype(np.float64)).astype(f)
        R_ = be * (V - up * (K @ once(S)))
        U = once(T) @ once(R_)
        out.append(up * (Q @ once(S)) + once(D * (Q @ K.T)) @ once(U))
        N = K.T @ twice(down * (twice(T) @ twice(be * up * K)))
        Z = K.T @ twice(down * (twice(T) @ twice(be * V)))
        S = whole * S + Z - twice(N) @ twice(S)
    return np.concatenate(out).astype(np.float64), S.astype(np.float64)


def test_the_bounds_tell_operands_of_fewer_bits(rng):
    def bf(x):
        return torch.from_numpy(np.ascontiguousarray(x)).bfloat16().float().numpy()

    def two(x):
        return bf(x) + bf(x - bf(x))

    x = _inputs(rng, 150, 64, 64, weak=0.5)
    x = [bf(t.astype(np.float32)).astype(np.float64) for t in x]
    O, S = R.delta_fwd(*x)
    worst = lambda y, ref, e: float((np.abs(y - ref) / (e + 2.0 ** -60)).max())  # noqa: E731
    b = R.delta_bounds(*x, None, 64, 2.0 ** -8, 2.0 ** -16)
    o, s = _chunked(*x, 64, bf, two)
    assert worst(o, O, b["O"]) <= 1 and worst(s, S, b["S_out"]) <= 1
    o, s = _chunked(*x, 64, bf, bf)
    assert worst(s, S, b["S_out"]) > 4                            # a state whose operands have one part
    b = R.delta_bounds(*x, None, 32, 0.0, 0.0)
    o, s = _chunked(*x, 32, lambda y: y, lambda y: y)
    assert worst(o, O, b["O"]) <= 1 and worst(s, S, b["S_out"]) <= 1
    o, s = _chunked(*x, 32, bf, two)
    assert worst(o, O, b["O"]) > 4


@pytest.mark.parametrize("gains", [True, False])
def test_layer_norm_gradient_against_differences(rng, gains):
    n, D = 3, 6
    X, Y = rng.normal(size=(n, D)) + 2, rng.normal(size=(n, D))
    w, b = (rng.normal(size=D), rng.normal(size=D)) if gains else (None, None)
    up, dN = rng.normal(size=(n, D)), rng.normal(size=(n, D))

    def loss():
        v, _ = R.layer_norm_fwd(X, Y, w, b)
        return (v["X_out"] * up).sum() + (v["N"] * dN).sum()

    after = R.layer_norm_fwd(X, Y, w, b)[0]["X_out"]
    v, m = R.layer_norm_bwd(after, dN, w, up)
    for k, t in (("dX", X), ("dX", Y), ("dw", w), ("db", b)):
        if t is not None:
            assert np.allclose(v[k], _differences(loss, t), rtol=1e-6, atol=1e-7), k
            assert (np.abs(v[k]) <= m[k] * (1 + 1e-12) + 1e-15).all(), k


# ------------------------------------------------------------------------------------------- refusals
A0, SZ = 0x10000, 1 << 40      # made-up aligned addresses far apart: every call below has to be refused (or be empty) before they are used
NULL, SHAPE, DIM, ALIGN, ALIAS, WS = -1, -2, -3, -5, -6, -7


def at(k):
    return A0 + k * SZ


@pytest.fixture(scope="module")
def L():
    from paper_2406_08128_amd import binding
    return binding.lib()


FORMS = [(form, sfx) for form in ("", "_cleared") for sfx in ("", "_f32")]


@pytest.mark.parametrize("form,sfx", FORMS)
def test_gated_delta_refusals(L, form, sfx):
    f = getattr(L, "chela_gated_delta_fwd" + form + sfx)

    def fwd(Q=at(0), ldq=128, K=at(1), ldk=128, V=at(2), ldv=256, g=at(3), ldg=4, beta=at(4), ldb=4, scale=1.0, cu=None, n_seq=2, T=8, H=4, Hk=2, dk=64,
            dv=64, S_in=at(5), S_out=at(6), slots=None, n_slots=2, O=at(7), saved=at(8)):
        return f(Q, ldq, K, ldk, V, ldv, g, ldg, beta, ldb, scale, cu, n_seq, T, H, Hk, dk, dv, S_in, S_out, slots, n_slots, O, saved, None)

    for n in ("Q", "K", "V", "beta", "O"):
        assert fwd(**{n: None}) == NULL, n
    for n in (0, 32, 96, 256):
        assert fwd(dk=n) == DIM and fwd(dv=n) == DIM
    assert fwd(H=-1) == SHAPE and fwd(Hk=0) == SHAPE and fwd(Hk=3) == SHAPE and fwd(Hk=-2) == SHAPE and fwd(H=1 << 15, Hk=1) == SHAPE
    for bad in (float("nan"), float("inf"), -float("inf")):
        assert fwd(scale=bad) == SHAPE
    assert fwd(T=-2) == SHAPE and fwd(T=7) == SHAPE and fwd(n_seq=-1) == SHAPE and fwd(n_seq=0, n_slots=0) == SHAPE and fwd(n_slots=3) == SHAPE
    assert fwd(ldq=127) == SHAPE and fwd(ldk=1) == SHAPE and fwd(ldv=255) == SHAPE and fwd(ldg=3) == SHAPE and fwd(ldb=0) == SHAPE
    assert fwd(ldv=1 << 29) == SHAPE
    assert fwd(T=1 << 24) == SHAPE and fwd(n_seq=1 << 19, T=1 << 19, n_slots=1 << 19) == SHAPE
    e = 1                                                     # (an element has 2 or 4 bytes: one off is none of either)
    for n, k in (("Q", 0), ("K", 1), ("V", 2), ("g", 3), ("beta", 4)):
        assert fwd(**{n: at(k) + e}) == ALIGN, n
    for n, k in (("S_in", 5), ("S_out", 6), ("O", 7), ("saved", 8)):
        assert fwd(**{n: at(k) + 8}) == ALIGN, n
    assert fwd(cu=at(9) + 2) == ALIGN and fwd(slots=at(9) + 1) == ALIGN
    for k in range(6):
        assert fwd(O=at(k)) == ALIAS and fwd(saved=at(k)) == ALIAS, k
        if k != 5:
            assert fwd(S_out=at(k)) == ALIAS
    assert fwd(S_out=at(5) + 16) == ALIAS and fwd(S_out=at(7)) == ALIAS and fwd(saved=at(7)) == ALIAS
    for n in ("Q", "K", "V", "g", "beta", "cu", "slots"):     # in place, and another input there
        assert fwd(**{n: at(5), "S_out": at(5)}) == ALIAS, n
    assert fwd(H=0, Hk=1) == 0 and fwd(T=0, n_seq=0, n_slots=0, Q=None, O=None) == 0
    b = getattr(L, "chela_gated_delta_bwd" + form + sfx)

    def bwd(Q=at(0), K=at(1), V=at(2), g=at(3), beta=at(4), scale=1.0, T=8, H=4, Hk=2, dk=64, dv=64, S_in=at(5), dO=at(6), lddo=256, dS_out=at(7),
            saved=at(8), dQ=at(9), dK=at(10), dV=at(11), dg=at(12), dbeta=at(13), dS_in=at(14)):
        return b(Q, 128, K, 128, V, 256, g, 4, beta, 4, scale, None, 2, T, H, Hk, dk, dv, S_in, dO, lddo, dS_out, saved, dQ, dK, dV, dg, dbeta, dS_in,
                 None)

    for n in ("Q", "K", "V", "beta", "dO", "dQ", "dK", "dV", "dg", "dbeta"):
        assert bwd(**{n: None}) == NULL, n
    assert bwd(dk=96) == DIM and bwd(dv=65) == DIM and bwd(Hk=3) == SHAPE and bwd(T=9) == SHAPE and bwd(lddo=255) == SHAPE and bwd(scale=float("nan")) == SHAPE
    for n, k in (("dQ", 9), ("dK", 10), ("dV", 11), ("dg", 12), ("dbeta", 13), ("dS_in", 14), ("saved", 8), ("dS_out", 7)):
        assert bwd(**{n: at(k) + 4}) == ALIGN, n
    for n in ("dQ", "dK", "dV", "dg", "dbeta", "dS_in"):
        for k in list(range(9)) + [9 if n != "dQ" else 10]:
            assert bwd(**{n: at(k)}) == ALIAS, (n, k)
    s = getattr(L, "chela_gated_delta_step" + form + sfx)

    def step(q=at(0), ldq=128, v=at(2), beta=at(4), scale=1.0, S=at(5), slots=None, n_slots=3, R=3, H=4, Hk=2, dk=64, dv=64, o=at(6)):
        return s(q, ldq, at(1), 128, v, 256, None, 0, beta, 4, scale, S, slots, n_slots, R, H, Hk, dk, dv, o, None)

    for n in ("q", "v", "beta", "S", "o"):
        assert step(**{n: None}) == NULL, n
    assert step(dk=63) == DIM and step(Hk=3) == SHAPE and step(R=-1) == SHAPE and step(n_slots=4) == SHAPE and step(ldq=5) == SHAPE
    assert step(R=1 << 21, n_slots=1 << 21) == SHAPE and step(scale=float("inf")) == SHAPE
    assert step(S=at(5) + 4) == ALIGN and step(o=at(6) + 2) == ALIGN
    assert step(o=at(5)) == ALIAS and step(S=at(0)) == ALIAS and step(o=at(2)) == ALIAS
    assert step(R=0, n_slots=0, q=None, S=None) == 0


@pytest.mark.parametrize("sfx", ["", "_f32"])
def test_layer_norm_refusals(L, sfx):
    f = getattr(L, "chela_layer_norm_fwd" + sfx)

    def fwd(X=at(0), Y=at(1), w=at(2), b=at(3), X_out=at(4), N=at(5), eps=1e-5, rows=4, D=64, x_f32=0):
        return f(X, Y, w, b, X_out, N, eps, rows, D, x_f32, None)

    assert fwd(X=None) == NULL and fwd(X_out=None) == NULL and fwd(N=None) == NULL and fwd(Y=None, N=None) == NULL
    assert fwd(rows=-1) == SHAPE and fwd(rows=1 << 31) == SHAPE and fwd(D=0) == SHAPE and fwd(D=8193) == DIM
    for bad in (float("nan"), float("inf"), -1.0):
        assert fwd(eps=bad) == SHAPE
    for n, k in (("X", 0), ("Y", 1), ("w", 2), ("b", 3), ("X_out", 4), ("N", 5)):
        assert fwd(**{n: at(k) + 8}) == ALIGN, n
    for k in range(1, 4):
        assert fwd(X_out=at(k)) == ALIAS and fwd(N=at(k)) == ALIAS
    assert fwd(N=at(0)) == ALIAS and fwd(N=at(4)) == ALIAS and fwd(X_out=at(0) + 16) == ALIAS
    assert fwd(X_out=at(0), w=at(0)) == ALIAS
    if sfx == "":
        assert fwd(X_out=at(0), Y=at(0), x_f32=1) == ALIAS        # (rows of another type: elements are elsewhere)
    assert fwd(rows=0, X=None, X_out=None, N=None) == 0
    g = getattr(L, "chela_layer_norm_bwd" + sfx)

    def bwd(X=at(0), w=at(1), up=at(2), dN=at(3), dX=at(4), dw=at(5), db=at(6), eps=1e-5, rows=4, D=64, x_f32=0):
        return g(X, w, up, dN, dX, dw, db, eps, rows, D, x_f32, None)

    assert bwd(X=None) == NULL and bwd(dN=None) == NULL and bwd(dX=None) == NULL
    assert bwd(rows=-2) == SHAPE and bwd(D=0) == SHAPE and bwd(D=9000) == DIM and bwd(eps=-1.0) == SHAPE
    for n, k in (("X", 0), ("w", 1), ("up", 2), ("dN", 3), ("dX", 4), ("dw", 5), ("db", 6)):
        assert bwd(**{n: at(k) + 8}) == ALIGN, n
    assert bwd(dX=at(0)) == ALIAS and bwd(dX=at(3)) == ALIAS and bwd(dw=at(6)) == ALIAS and bwd(db=at(1)) == ALIAS and bwd(dX=at(2) + 16) == ALIAS
    assert bwd(up=None, dX=at(0)) == ALIAS and bwd(dX=at(2), w=at(2)) == ALIAS


def test_workspace_and_saved_queries(L):
    saved, ws = L.chela_gated_delta_saved_bytes, L.chela_gated_delta_workspace_bytes
    for bad in ((0, 1, 0, 2, 64, 64, 0), (10, 3, 0, 2, 64, 64, 0), (10, 0, 1, 2, 64, 64, 0), (64, 1, 0, 2, 32, 64, 0), (64, 1, 0, 0, 64, 64, 0),
                (1 << 27, 1, 0, 16, 64, 64, 0)):
        assert saved(*bad) == 0, bad
        assert ws(*bad, 0, 0) == 0 and ws(*bad, 1, 1) == 0, bad
    # per chunk and head: the inverse and the state in bf16; the transition in two parts, the state's part in fp32, e^gamma
    assert saved(128, 1, 0, 1, 64, 64, 0) == 2 * (64 * 64 * 2 + 64 * 64 * 2)
    assert ws(128, 1, 0, 1, 64, 64, 0, 0, 1) == 2 * (2 * 64 * 64 * 2 + 64 * 64 * 4) + 256
    assert ws(128, 1, 0, 1, 64, 64, 0, 0, 0) == ws(128, 1, 0, 1, 64, 64, 0, 0, 1) + saved(128, 1, 0, 1, 64, 64, 0)
    assert saved(128, 4, 1, 2, 64, 128, 1) > saved(128, 1, 1, 2, 64, 128, 1) > saved(128, 1, 0, 2, 64, 128, 1) > 0
    assert ws(128, 1, 0, 1, 64, 64, 0, 1, 1) > ws(128, 1, 0, 1, 64, 64, 0, 0, 1)
    assert L.chela_layer_norm_bwd_workspace_bytes(10, 64) > 0 and L.chela_layer_norm_bwd_workspace_bytes(10, 8193) == 0
    assert L.chela_layer_norm_bwd_workspace_bytes(-1, 64) == 0


def test_a_workspace_that_is_too_small_is_refused(L):
    L.chela_set_workspace(A0, 256)
    try:
        row = (at(0), 64, at(1), 64, at(2), 64, None, 0, at(3), 1, 1.0)
        assert L.chela_gated_delta_fwd(*row, None, 1, 8, 1, 1, 64, 64, None, None, None, 1, at(4), None, None) == WS
        assert L.chela_gated_delta_bwd(*row, None, 1, 8, 1, 1, 64, 64, None, at(4), 64, None, None, at(5), at(6), at(7), None, at(8), None, None) == WS
        assert L.chela_layer_norm_bwd(at(0), at(1), None, at(2), at(3), at(4), None, 1e-5, 4, 64, 0, None) == WS
    finally:
        L.chela_set_workspace(None, 0)


def test_the_places_of_chunks():
    # sequence s's chunks begin at cu[s] / C + s: no two sequences share a place and T / C + n_seq are enough, whatever the lengths
    r = np.random.default_rng(5)
    for C in (32, 64):
        for _ in range(200):
            lens = r.integers(0, 3 * C, size=r.integers(1, 9)) * (r.random() < 0.8)
            lens[r.integers(len(lens))] += r.integers(0, 2)
            first = int(r.integers(0, 2 * C))
            cu = np.concatenate([[first], first + np.cumsum(lens)])
            T = int(cu[-1] + r.integers(0, C))
            at_ = cu[:-1] // C + np.arange(len(lens))
            end = at_ + -(-lens // C)
            assert (end[:-1] <= at_[1:]).all() and end[-1] <= T // C + len(lens)


def test_binding_refuses_what_it_cannot_hand_on():
    from paper_2406_08128_amd import binding
    q, b, x = torch.zeros(4, 2, 64), torch.zeros(4, 2), torch.zeros(4, 8)
    with pytest.raises(ValueError):
        binding.chela_gated_delta_fwd(q, q, q, None, b)              # not on a device
    with pytest.raises(ValueError):
        binding.chela_gated_delta_bwd(q, q, q, None, b, q)
    with pytest.raises(ValueError):
        binding.chela_gated_delta_step(q, q, q, None, b, torch.zeros(4, 2, 64, 64))
    with pytest.raises(ValueError):
        binding.chela_layer_norm_fwd(x)
    with pytest.raises(ValueError):
        binding.chela_layer_norm_bwd(x, x)


@pytest.mark.parametrize("form,sfx", FORMS)
def test_the_walk_of_the_states_stays_below_2_to_the_32_threads(L, form, sfx):
    # eight workgroups at a time, of 4 dk threads, one for sixteen columns of a state: 2^21 - 1 states of 128 x 64 would be 2^32 threads
    n, dtype = (1 << 21) - 1, int(sfx == "_f32")
    for m, ok in ((n - 1, True), (n, False)):
        got = [L.chela_gated_delta_workspace_bytes(64, m, 1, 1, 128, 64, dtype, b, 0) for b in (0, 1)] + [L.chela_gated_delta_saved_bytes(64, m, 1, 1, 128, 64, dtype)]
        assert all((x > 0) == ok for x in got)
    x = (at(0), 128, at(1), 128, at(2), 64, None, 0, at(3), 1, 1.0, at(4), n, 64, 1, 1, 128, 64)
    assert getattr(L, "chela_gated_delta_fwd" + form + sfx)(*x, None, None, None, n, at(5), None, None) == SHAPE
    assert getattr(L, "chela_gated_delta_bwd" + form + sfx)(*x, None, at(5), 64, None, None, at(6), at(7), at(8), None, at(9), None, None) == SHAPE
