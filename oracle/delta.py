"""The gated delta rule and the layer norm with its residual in 64 bits: definitions, gradients, and bounds of what rounding may change.

Delta rule, one head: S' = e^g S, u = beta (v - S'^T k), S = S' + k u^T, o = scale S^T q; q, k [L, dk], v [L, dv], g, beta [L],
S [dk, dv].  Nothing here uses chunks but `delta_bounds`, which says by how much a computation in chunks may be off."""
import numpy as np


def delta_fwd(q, k, v, g, beta, scale=1.0, state=None):
    """(O, S_out)"""
    S = np.zeros((k.shape[1], v.shape[1])) if state is None else state
    a = np.ones(len(k)) if g is None else np.exp(g)
    O = np.zeros(v.shape)
    for t in range(len(k)):
        S = a[t] * S
        S = S + np.outer(k[t], beta[t] * (v[t] - k[t] @ S))
        O[t] = scale * (q[t] @ S)
    return O, S


def delta_bwd(q, k, v, g, beta, dO, scale=1.0, state=None, dstate=None):
    """{dQ, dK, dV, dg, dbeta, dS_in}"""
    L = len(k)
    states = [np.zeros((k.shape[1], v.shape[1])) if state is None else state]
    a = np.ones(L) if g is None else np.exp(g)
    for t in range(L):
        S = a[t] * states[-1]
        states.append(S + np.outer(k[t], beta[t] * (v[t] - k[t] @ S)))
    out = {"dQ": np.zeros(q.shape), "dK": np.zeros(k.shape), "dV": np.zeros(v.shape), "dg": np.zeros(L), "dbeta": np.zeros(L)}
    G = np.zeros(states[0].shape) if dstate is None else dstate            # of the state behind a token
    for t in range(L - 1, -1, -1):
        before = a[t] * states[t]
        e = v[t] - k[t] @ before
        out["dQ"][t] = scale * (states[t + 1] @ dO[t])
        G = G + scale * np.outer(q[t], dO[t])
        du = k[t] @ G
        out["dbeta"][t] = du @ e
        out["dV"][t] = beta[t] * du
        out["dK"][t] = G @ (beta[t] * e) - before @ out["dV"][t]
        G = G - np.outer(k[t], out["dV"][t])
        out["dg"][t] = (G * before).sum()
        G = a[t] * G
    out["dS_in"] = G
    return out


# ---- bounds.  A quantity is a pair (value, what it may be off by); a product's terms are each off by what their factors are off by, and n of them
# are added up in fp32.

F = 2.0 ** -24


def _mm(a, b):
    (x, dx), (y, dy) = a, b
    return x @ y, np.abs(x) @ dy + dx @ (np.abs(y) + dy) + (x.shape[1] + 2) * F * (np.abs(x) @ np.abs(y))


def _times(a, f, rel=4 * F):
    x, dx = a
    return x * f, (dx + rel * np.abs(x)) * np.abs(f)


def _plus(a, b):
    return a[0] + b[0], a[1] + b[1] + F * (np.abs(a[0]) + np.abs(b[0]))


def _onto(a, b, n):
    """A product b of n terms that are added to a one by one: each sum is rounded, a in it."""
    return a[0] + b[0], a[1] + b[1] + (n + 2) * F * (np.abs(a[0]) + np.abs(b[0]))


def _rounded(a, u):
    return a[0], a[1] + u * (np.abs(a[0]) + a[1])


def _t(a):
    return a[0].T, a[1].T


def _exact(x):
    return x, np.zeros(x.shape)


def delta_bounds(q, k, v, g, beta, dO, chunk, once, twice, scale=1.0, state=None, dstate=None):
    """What O, S_out and the gradients may be off by before they are rounded themselves.  once: half a step of an operand of a matrix product that is
    rounded, twice: of one that has two parts (0 where operands keep fp32).  An error of a state that goes through a chunk is at most as large
    as its columns' norm times the largest singular value of what the chunk makes of a state; everything else is element by element."""
    L, dk, dv = len(k), k.shape[1], v.shape[1]
    g = np.zeros(L) if g is None else np.maximum(g, -256.0)
    spans = [(a, min(a + chunk, L)) for a in range(0, L, chunk)]
    zero = np.zeros((dk, dv))
    S = _exact(zero if state is None else state)
    parts = []

    def walk(M, whole, S, Z, N):
        # whole S + Z - N S, N and S in two parts.  (whole = e^gamma is off as the other exponentials are: its argument gamma log2 e by two
        # roundings, 2 F |gamma|, and itself by the exponential's last digit, 2 F; its product and the sum, 2 F, on top: no more than 8 F (1 + |gamma|).
        # The dk terms of N S are added to whole S + Z one by one, and each such sum is rounded as a whole.)
        local = (Z[1] + N[1] @ np.abs(S[0]) + (2 * twice + (dk + 4) * F) * (np.abs(N[0]) @ np.abs(S[0])) +
                 8 * F * (1 - np.log(max(whole, 1e-100))) * np.abs(whole * S[0]) + (dk + 4) * F * (np.abs(whole * S[0]) + np.abs(Z[0])))
        value = M @ S[0] + Z[0]
        norm = np.linalg.norm(M, 2) * np.sqrt((S[1] ** 2).sum(0)) + np.sqrt((local ** 2).sum(0))
        return value, np.minimum(np.abs(M) @ S[1] + local, norm[None, :] * np.ones((dk, 1)))

    for a, b in spans:
        n = b - a
        gamma = np.cumsum(g[a:b])
        D = np.tril(np.exp(np.tril(gamma[:, None] - gamma[None, :])))
        erel = 8 * F * (1 + np.abs(gamma[:, None] - gamma[None, :]))
        up, down, whole = np.exp(gamma)[:, None], np.exp(gamma[-1] - gamma)[:, None], np.exp(gamma[-1])
        grel = 8 * F * (1 + np.abs(gamma))[:, None]
        K, Q, V, be = k[a:b], q[a:b], v[a:b], beta[a:b, None]
        G = _mm(_exact(K), _exact(K.T))
        A = np.tril(be * D * G[0], -1)
        dA = np.tril(be * D * G[1], -1) + np.abs(A) * erel
        T = np.linalg.inv(np.eye(n) + A)
        T = (T, np.abs(T) @ (dA + (n + 4) * F * (np.abs(A) + np.eye(n))) @ np.abs(T))
        T2 = _rounded(T, twice)
        W = _mm(T2, _rounded(_times(_exact(K), be * up, grel), twice))
        U0 = _mm(T2, _rounded(_times(_exact(V), be), twice))
        N = _rounded(_mm(_exact(K.T), _rounded(_times(W, down, grel), twice)), twice)
        Z = _mm(_exact(K.T), _rounded(_times(U0, down, grel), twice))
        M = whole * np.eye(dk) - N[0]
        parts.append(dict(a=a, b=b, D=D, erel=erel, up=up, down=down, grel=grel, whole=whole, K=K, Q=Q, V=V, be=be, T2=T2, T1=_rounded(T, once), N=N, M=M,
                          S=_rounded(S, once), G=G))
        S = walk(M, whole, S, Z, N)
    out = {"S_out": S[1], "O": np.zeros((L, dv))}
    for p in parts:
        KS = _times(_mm(_exact(p["K"]), p["S"]), p["up"], p["grel"])
        R = _times(_plus(_exact(p["V"]), (-KS[0], KS[1])), p["be"])
        p["U"] = _mm(p["T1"], _rounded(R, once))
        P = _mm(_exact(p["Q"]), _exact(p["K"].T))
        p["QK"], p["P"] = P, _times(P, scale * p["D"], p["erel"])
        QS = _times(_mm(_exact(p["Q"]), p["S"]), scale * p["up"], p["grel"])
        out["O"][p["a"]:p["b"]] = _onto(QS, _mm(_rounded(p["P"], once), _rounded(p["U"], once)), p["b"] - p["a"])[1]
    if dO is None:
        return out
    out.update(dQ=np.zeros(q.shape), dK=np.zeros(k.shape), dV=np.zeros(v.shape), dg=np.zeros(L), dbeta=np.zeros(L), dg_sums=np.zeros(L), dg_divided=np.zeros(L))
    dS = _exact(zero if dstate is None else dstate)
    for p in parts[::-1]:
        a, b, K, Q, be, up, down, grel, D, erel = (p[x] for x in ("a", "b", "K", "Q", "be", "up", "down", "grel", "D", "erel"))
        d = dO[a:b]
        # the gradients, from the state's behind
        B = _rounded(dS, once)
        dU = _onto(_times(_mm(_exact(K), B), down, grel), _mm(_t(_rounded(p["P"], once)), _exact(d)), b - a)
        dR = _mm(_t(p["T1"]), _rounded(dU, once))
        out["dV"][a:b] = _times(dR, be)[1]
        R, U = _rounded(dR, once), _rounded(p["U"], once)
        X = _times(_mm(_exact(d), _t(U)), scale * D, erel)
        Y = _times(_mm(R, _t(U)), np.tril(D, -1), erel)
        Yb = _rounded(_times(Y, be), once)
        X1 = _rounded(X, once)
        dQ = _onto(_times(_mm(_exact(d), _t(p["S"])), scale * up, grel), _mm(X1, _exact(K)), b - a)
        into = _times(_mm(R, _t(p["S"])), up, grel)
        read = _onto(_times(into, be), _mm(Yb, _exact(K)), b - a)
        carry = _times(_mm(U, _t(B)), down, grel)
        pairs = _mm(_t(Yb), _exact(K))
        write = _plus(_onto(carry, _mm(_t(X1), _exact(Q)), b - a), (-pairs[0], pairs[1]))
        out["dQ"][a:b], out["dK"][a:b] = dQ[1], _plus((-read[0], read[1]), write)[1]

        def dot(x, y, size):
            return (np.abs(x) * (y[1] + (size + 4) * F * np.abs(y[0]))).sum(1)

        out["dbeta"][a:b] = dot(p["V"], dR, dv) + dot(K, into, dk) + dot(Y[0], p["G"], b - a) + (Y[1] * np.abs(p["G"][0])).sum(1)
        # Decays: a pair of tokens on one side of t goes into dgamma twice, from the same rounded X and Y, and cancels but for sums' roundings (512
        # of them on any way); what X and Y are off by comes in through the pairs that t divides.
        QK = np.abs(p["QK"][0])
        pair = X1[1] * QK + Yb[1] * np.abs(p["G"][0])
        size = np.abs(X1[0]) * QK + np.abs(Yb[0]) * np.abs(p["G"][0])
        oS = _times(_mm(_exact(d), _t(p["S"])), scale * up, grel)
        near, far = dot(Q, oS, dk) + dot(K, _times(into, be), dk), dot(K, carry, dk)
        SB = (np.abs(p["S"][0]) * (B[1] + dk * F * np.abs(B[0])) + p["S"][1] * np.abs(B[0])).sum()
        sums = size.sum() + (np.abs(Q * oS[0]) + np.abs(K * into[0] * be) + np.abs(K * carry[0])).sum() + p["whole"] * np.abs(p["S"][0] * B[0]).sum()
        for t in range(b - a):
            out["dg_sums"][a + t] = 512 * F * sums              # (of it what is left where all of it cancels, a first token's without a state)
            out["dg"][a + t] = pair[t:, :t].sum() + near[t:].sum() + far[:t].sum() + p["whole"] * SB + 512 * F * sums
        # ... and where only the pairs that t divides are added up, with what comes from the state in front to t and later tokens, what tokens in front of t
        # hand to the one behind, and what goes through: each term has the factor e^g_t, so the bound has it too.  X and Y need not be rounded for it.
        Ye = _times(Y, be)
        pair = X[1] * QK + np.abs(X[0]) * p["QK"][1] + Ye[1] * np.abs(p["G"][0]) + np.abs(Ye[0]) * p["G"][1]
        size = np.abs(X[0]) * QK + np.abs(Ye[0]) * np.abs(p["G"][0])
        onear, ofar = np.abs(Q * oS[0]).sum(1) + np.abs(K * into[0] * be).sum(1), np.abs(K * carry[0]).sum(1)
        through = p["whole"] * np.abs(p["S"][0] * B[0]).sum()
        for t in range(b - a):
            mags = size[t:, :t].sum() + onear[t:].sum() + ofar[:t].sum() + through * (1 + abs(np.log(max(p["whole"], 1e-100))))
            out["dg_divided"][a + t] = pair[t:, :t].sum() + near[t:].sum() + far[:t].sum() + p["whole"] * SB + (2 * (b - a) + 32) * F * mags
        # and of the state in front
        x = _rounded(_mm(_t(_rounded(p["P"], twice)), _exact(d)), twice)
        y = _rounded(_times(_mm(_t(p["T2"]), x), be * up, grel), twice)
        z = _mm(_exact(K.T), y)
        Zb = _onto(_mm(_exact(Q.T), _rounded(_times(_exact(d), scale * up, grel), twice)), (-z[0], z[1]), b - a)
        dS = walk(p["M"].T, p["whole"], dS, Zb, _t(p["N"]))
    out["dS_in"] = dS[1]
    return out


# ---- layer norm: X' = X + Y, N = (X' - m) s w + b

def layer_norm_fwd(X, Y=None, w=None, b=None, eps=1e-5):
    """({X_out, N}, masses)"""
    after, ma = (X, np.abs(X)) if Y is None else (X + Y, np.abs(X) + np.abs(Y))
    m = after.mean(-1, keepdims=True)
    s = 1.0 / np.sqrt(((after - m) ** 2).mean(-1, keepdims=True) + eps)
    n = (after - m) * s
    w = np.ones(X.shape[-1]) if w is None else w
    # (what the row is off by, the mean among it, reaches n itself and, by half of the sum of squares' relative error, through s)
    md = s * (ma + np.abs(after).mean(-1, keepdims=True))
    mass = np.abs(w) * (md + np.abs(n) * (1 + (md * np.abs(n)).mean(-1, keepdims=True))) + (0 if b is None else np.abs(b))
    return {"X_out": after, "N": n * w + (0 if b is None else b)}, {"X_out": ma, "N": mass}


def layer_norm_bwd(X_out, dN, w=None, dX_out=None, eps=1e-5):
    """({dX, dw, db}, masses) from the stream as the forward call left it."""
    c = X_out - X_out.mean(-1, keepdims=True)
    s = 1.0 / np.sqrt((c ** 2).mean(-1, keepdims=True) + eps)
    n = c * s
    w = np.ones(X_out.shape[-1]) if w is None else w
    v, mv = dN * w, np.abs(dN * w)
    mean = lambda x: x.mean(-1, keepdims=True)  # noqa: E731
    dx = s * (v - mean(v) - n * mean(v * n))
    mn = s * (np.abs(X_out) + mean(np.abs(X_out)))                 # of n
    mn = mn + np.abs(n) * (1 + mean(mn * np.abs(n)))
    mx = s * (mv + mean(mv) + mn * mean(mv * np.abs(n)) + np.abs(n) * mean(mv * mn)) + np.abs(dx) * (1 + mean(mn * np.abs(n)))
    flat = lambda x: x.reshape(-1, x.shape[-1])  # noqa: E731
    up, mup = (0, 0) if dX_out is None else (dX_out, np.abs(dX_out))
    return ({"dX": dx + up, "dw": flat(dN * n).sum(0), "db": flat(dN).sum(0)},
            {"dX": mx + mup, "dw": flat(np.abs(dN) * mn).sum(0), "db": flat(np.abs(dN)).sum(0)})
