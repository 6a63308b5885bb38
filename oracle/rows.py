"""Definitions, in 64 bits and token by token, of the operators on rows: the short causal convolution, the selective scan and the norms
around a block, with their gradients.

Every function returns, beside each value, its mass: the same sum with every term's magnitude in the place of the term.  A kernel that adds n
rounded terms in fp32 is off by no more than about n 2^-24 times the mass, however much of it cancels: tolerance() says so.

A sequence is [L, D]; packed rows are taken apart by the caller.
"""
import numpy as np


def sigmoid(x):
    return 1.0 / (1.0 + np.exp(-x))


def silu(x):
    return x * sigmoid(x)


def dsilu(x):
    """(silu', mass of it)"""
    s = sigmoid(x)
    return s * (1 + x * (1 - s)), s * (1 + np.abs(x) * (1 - s))


def tolerance(ref, mass, n, half_step):
    """|got - ref| for an output rounded once to a type of that half step (relative), after at most n fp32 roundings of the mass.
    (1e-30: results that fp32 flushes.)"""
    err = n * 2.0 ** -24 * mass
    return half_step * (np.abs(ref) + err) + err + 1e-30


# ---- short causal convolution: u_t = bias + sum_j w[:, j] x_{t-j}, y = silu(u) or u

def short_conv_fwd(x, w, bias=None, act=True, state=None):
    """(y, mass, state behind) of x [L, D], w [D, m], state [m-1, D] (the last inputs in front, the latest last)."""
    L, D = x.shape
    m = w.shape[1]
    ext = np.concatenate([np.zeros((m - 1, D)) if state is None else state, x])
    b = np.zeros(D) if bias is None else bias
    u, mu = np.tile(b, (L, 1)), np.tile(np.abs(b), (L, 1))
    for j in range(m):
        u = u + w[:, j] * ext[m - 1 - j:m - 1 - j + L]
        mu = mu + np.abs(w[:, j] * ext[m - 1 - j:m - 1 - j + L])
    if not act:
        return u, mu, ext[L:]
    # (an error of u's mass reaches y through |silu'| <= 1.1, and the activation's own through |u|)
    return silu(u), 1.1 * mu + np.abs(u), ext[L:]


def short_conv_bwd(x, w, dy, bias=None, act=True, state=None, dstate=None):
    """({dX, dw, dbias, dS_in}, masses) for the upstream dy [L, D] and dstate [m-1, D]."""
    L, D = x.shape
    m = w.shape[1]
    ext = np.concatenate([np.zeros((m - 1, D)) if state is None else state, x])
    b = np.zeros(D) if bias is None else bias
    u, mu = np.tile(b, (L, 1)), np.tile(np.abs(b), (L, 1))
    for j in range(m):
        u = u + w[:, j] * ext[m - 1 - j:m - 1 - j + L]
        mu = mu + np.abs(w[:, j] * ext[m - 1 - j:m - 1 - j + L])
    if act:
        d, dm = dsilu(u)
        du, mdu = dy * d, np.abs(dy) * (dm + 0.6 * mu)          # |silu''| <= 0.5
    else:
        du, mdu = dy, np.abs(dy)
    dext, mext = np.zeros((L + m - 1, D)), np.zeros((L + m - 1, D))
    dw, mw = np.zeros((D, m)), np.zeros((D, m))
    for j in range(m):
        at = slice(m - 1 - j, m - 1 - j + L)
        dext[at] += w[:, j] * du
        mext[at] += np.abs(w[:, j]) * mdu
        dw[:, j] = (du * ext[at]).sum(0)
        mw[:, j] = (mdu * np.abs(ext[at])).sum(0)
    if dstate is not None and m > 1:
        dext[L:] += dstate
        mext[L:] += np.abs(dstate)
    return ({"dX": dext[m - 1:], "dw": dw, "dbias": du.sum(0), "dS_in": dext[:m - 1]},
            {"dX": mext[m - 1:], "dw": mw, "dbias": mdu.sum(0), "dS_in": mext[:m - 1]})


# ---- selective scan: h[n] = exp(dl A[n]) h[n] + dl u B[n], y = sum_n C[n] h[n] + D u, out = y silu(z)

def _scan_setup(delta, A, Bm, Cm, delta_bias, softplus, D):
    raw = delta if delta_bias is None else delta + delta_bias
    dl = np.logaddexp(0.0, raw) if softplus else raw
    per = D // Bm.shape[1]
    return raw, dl, np.repeat(Bm, per, axis=1).transpose(0, 2, 1), np.repeat(Cm, per, axis=1).transpose(0, 2, 1)


def selscan_fwd(u, delta, A, Bm, Cm, skip=None, z=None, delta_bias=None, softplus=True, state=None):
    """({Y, S_out}, masses) of u, delta, z [L, D], A [N, D], Bm, Cm [L, G, N], skip, delta_bias [D], state [N, D]."""
    L, D = u.shape
    raw, dl, Be, Ce = _scan_setup(delta, A, Bm, Cm, delta_bias, softplus, D)
    h = np.zeros(A.shape) if state is None else state.copy()
    m = np.abs(h)
    y, my = np.zeros((L, D)), np.zeros((L, D))
    for t in range(L):
        a = np.exp(dl[t] * A)
        b = dl[t] * u[t] * Be[t]
        h = a * h + b
        m = a * m + np.abs(b)
        y[t] = (Ce[t] * h).sum(0)
        my[t] = (np.abs(Ce[t]) * m).sum(0)
    if skip is not None:
        y = y + skip * u
        my = my + np.abs(skip * u)
    if z is not None:
        y, my = y * silu(z), my * np.abs(silu(z)) * (1 + 0.1 * np.abs(z))
    return {"Y": y, "S_out": h}, {"Y": my, "S_out": m}


def selscan_bwd(u, delta, A, Bm, Cm, dY, skip=None, z=None, delta_bias=None, softplus=True, state=None, dstate=None):
    """({dU, ddelta, dA, dB, dC, dD, dZ, dbias, dS_in}, masses)."""
    L, D = u.shape
    N, G = A.shape[0], Bm.shape[1]
    raw, dl, Be, Ce = _scan_setup(delta, A, Bm, Cm, delta_bias, softplus, D)
    first = np.zeros(A.shape) if state is None else state
    sk = np.zeros(D) if skip is None else skip
    hs, ms = [first], [np.abs(first)]
    y, my = np.zeros((L, D)), np.zeros((L, D))
    for t in range(L):
        a, b = np.exp(dl[t] * A), dl[t] * u[t] * Be[t]
        hs.append(a * hs[-1] + b)
        ms.append(a * ms[-1] + np.abs(b))
        y[t] = (Ce[t] * hs[-1]).sum(0) + sk * u[t]
        my[t] = (np.abs(Ce[t]) * ms[-1]).sum(0) + np.abs(sk * u[t])
    v = {k: np.zeros((L, D)) for k in ("dU", "ddelta", "dZ")}
    m = {k: np.zeros((L, D)) for k in ("dU", "ddelta", "dZ")}
    if z is not None:
        d, dm = dsilu(z)
        v["dZ"], m["dZ"] = dY * y * d, np.abs(dY) * my * dm * (1 + 0.1 * np.abs(z))
        dy, mdy = dY * silu(z), np.abs(dY * silu(z)) * (1 + 0.1 * np.abs(z))
    else:
        dy, mdy = dY, np.abs(dY)
    v["dB"], v["dC"], m["dB"], m["dC"] = (np.zeros((L, G, N)) for _ in range(4))
    v["dA"], m["dA"] = np.zeros(A.shape), np.zeros(A.shape)
    q = np.zeros(A.shape) if dstate is None else dstate
    mq = np.abs(q)
    groups = lambda x: x.reshape(N, G, D // G).sum(2).T  # noqa: E731
    for t in range(L - 1, -1, -1):
        a = np.exp(dl[t] * A)
        g, mg = Ce[t] * dy[t] + q, np.abs(Ce[t]) * mdy[t] + mq
        v["dC"][t], m["dC"][t] = groups(dy[t] * hs[t + 1]), groups(mdy[t] * ms[t + 1])
        v["dB"][t], m["dB"][t] = groups(g * dl[t] * u[t]), groups(mg * np.abs(dl[t] * u[t]))
        q, mq = a * g, a * mg
        p, mp = q * hs[t], mq * ms[t]
        v["dA"] += dl[t] * p
        m["dA"] += np.abs(dl[t]) * mp
        s1, ms1 = (g * Be[t]).sum(0), (mg * np.abs(Be[t])).sum(0)
        v["dU"][t], m["dU"][t] = dl[t] * s1 + sk * dy[t], np.abs(dl[t]) * ms1 + np.abs(sk) * mdy[t]
        f = sigmoid(raw[t]) if softplus else 1.0
        v["ddelta"][t] = f * (u[t] * s1 + (A * p).sum(0))
        m["ddelta"][t] = f * (np.abs(u[t]) * ms1 + (np.abs(A) * mp).sum(0)) * (1 + 0.1 * np.abs(raw[t]))
    v["dS_in"], m["dS_in"] = q, mq
    v["dD"], m["dD"] = (dy * u).sum(0), (mdy * np.abs(u)).sum(0)
    v["dbias"], m["dbias"] = v["ddelta"].sum(0), m["ddelta"].sum(0)
    return v, m


def selscan_roundings(u, delta, A, Bm, Cm, dY, skip=None, z=None, delta_bias=None, softplus=True, state=None, dstate=None, once=128):
    """For the outputs of selscan_fwd and selscan_bwd (but dA, dD, dbias): the sum over an output's terms of their magnitudes, each times the fp32
    roundings that it goes through.  Times 2^-24 that is what the output may be off by, and it says more than the longest sequence's
    roundings for all of them: a term that the decay has ended counts no more.

    A row that a term passes costs it, walked row by row, the exponent's product (4 |x|, x = dl A, with what dl and A log2 e are off by), the
    exponential and a multiply-add: 4 + 4 |x|.  Taken together with 24 other rows, and 32 such lots with one another, x is a part of a sum of step
    sizes whose 56 additions are each off by half a step of the sum: 60 |x| on top.  So 8 + 64 |x|.  once: for what is not passed from row
    to row, the input's products, the sum over at most 32 states, the activations."""
    L, D = u.shape
    N, G = A.shape[0], Bm.shape[1]
    raw, dl, Be, Ce = _scan_setup(delta, A, Bm, Cm, delta_bias, softplus, D)
    sk = np.zeros(D) if skip is None else np.abs(skip)
    ms, ks = [np.zeros(A.shape) if state is None else np.abs(state)], [np.zeros(A.shape)]
    out = {k: np.zeros((L, D)) for k in ("Y", "dU", "ddelta")}
    for t in range(L):
        a, w, b = np.exp(dl[t] * A), 8 + 64 * np.abs(dl[t] * A), np.abs(dl[t] * u[t] * Be[t])
        ks.append(a * (ks[-1] + w * ms[-1]) + once * b)
        ms.append(a * ms[-1] + b)
        out["Y"][t] = (np.abs(Ce[t]) * (ks[-1] + once * ms[-1])).sum(0) + once * sk * np.abs(u[t])
    out["S_out"] = ks[-1] + once * ms[-1]
    mdy = np.abs(dY)
    if z is not None:
        gate = np.abs(silu(z)) * (1 + 0.1 * np.abs(z))
        out["dZ"] = mdy * out["Y"] * dsilu(z)[1] * (1 + 0.1 * np.abs(z))
        out["Y"], mdy = out["Y"] * gate, mdy * gate
    out["dB"], out["dC"] = np.zeros((L, G, N)), np.zeros((L, G, N))
    mq = np.zeros(A.shape) if dstate is None else np.abs(dstate)
    kq = np.zeros(A.shape)
    groups = lambda x: x.reshape(N, G, D // G).sum(2).T  # noqa: E731
    for t in range(L - 1, -1, -1):
        a, w = np.exp(dl[t] * A), 8 + 64 * np.abs(dl[t] * A)
        mg, kg = np.abs(Ce[t]) * mdy[t] + mq, once * np.abs(Ce[t]) * mdy[t] + kq
        out["dC"][t] = groups(mdy[t] * (ks[t + 1] + (once + D) * ms[t + 1]))
        out["dB"][t] = groups((kg + (once + D) * mg) * np.abs(dl[t] * u[t]))
        kq, mq = a * (kg + w * mg), a * mg
        s1 = ((kg + once * mg) * np.abs(Be[t])).sum(0)
        out["dU"][t] = np.abs(dl[t]) * s1 + once * sk * mdy[t]
        f = (sigmoid(raw[t]) if softplus else 1.0) * (1 + 0.1 * np.abs(raw[t]))
        out["ddelta"][t] = f * (np.abs(u[t]) * s1 + (np.abs(A) * (kq * ms[t] + mq * ks[t] + once * mq * ms[t])).sum(0))
    out["dS_in"] = kq + once * mq
    return out


# ---- norms around a block: X' = X + scale Norm(Y) w_post gate, N = Norm(X') w_pre

def _norm(x, eps):
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    return x * r, r


def block_norm_fwd(Y, X, gate=None, w_post=None, w_pre=None, scale=1.0, eps=1e-5):
    """({X_out, N}, masses); Y None: N alone, of X."""
    after, ma = X, np.abs(X)
    if Y is not None:
        p = _norm(Y, eps)[0] * w_post if w_post is not None else Y
        p = scale * (p * gate if gate is not None else p)
        after, ma = X + p, np.abs(X) + np.abs(p)
    out, mass = {"X_out": after}, {"X_out": ma}
    if w_pre is not None:
        n, r = _norm(after, eps)
        # (a relative error of the sum of squares is one of at most twice mass over value, half of which reaches n)
        out["N"] = n * w_pre
        mass["N"] = np.abs(w_pre) * (r * ma + np.abs(n) * (1 + r * r * (ma * np.abs(after)).mean(-1, keepdims=True)))
    return out, mass


def block_norm_bwd(Y, X_out, dX_out, dN, gate=None, w_post=None, w_pre=None, scale=1.0, eps=1e-5):
    """({dY, dgate, dX, dw_post, dw_pre}, masses) from the stream as the forward call left it."""
    v, m = {}, {}
    dx, mx = (np.zeros(X_out.shape), np.zeros(X_out.shape)) if dX_out is None else (dX_out, np.abs(dX_out))

    def through(g, mg, x):
        n, r = _norm(x, eps)
        return (r * (g - n * (g * n).mean(-1, keepdims=True)),
                r * (2 * mg + 3 * np.abs(n) * (mg * np.abs(n)).mean(-1, keepdims=True)), n)

    if w_pre is not None:
        d, md, n = through(dN * w_pre, np.abs(dN * w_pre), X_out)
        dx, mx = dx + d, mx + md
        v["dw_pre"], m["dw_pre"] = (dN * n).reshape(-1, n.shape[-1]).sum(0), 2 * np.abs(dN * n).reshape(-1, n.shape[-1]).sum(0)
    v["dX"], m["dX"] = dx, mx
    if Y is not None:
        g = gate if gate is not None else np.ones(Y.shape)
        w = w_post if w_post is not None else np.ones(Y.shape[-1])
        dp, mp = scale * dx, abs(scale) * mx
        if w_post is not None:
            v["dY"], m["dY"], n = through(dp * w * g, mp * np.abs(w * g), Y)
            v["dw_post"] = (dp * n * g).reshape(-1, n.shape[-1]).sum(0)
            m["dw_post"] = 2 * (mp * np.abs(n * g)).reshape(-1, n.shape[-1]).sum(0)
        else:
            n = Y
            v["dY"], m["dY"] = dp * g, mp * np.abs(g)
        if gate is not None:
            v["dgate"], m["dgate"] = dp * n * w, 2 * mp * np.abs(n * w)
    return v, m
