"""The selective state space block's operators as cases that can be timed and compared: its short causal convolution, its
selective scan, and the norms around a block with their gate and residual.

Tokens are rows and channels are fastest, [T, D]; the T rows belong to sequences of one length each, or of the lengths that
the offsets `cu` give.  `listed()` holds fixed sizes (inner widths are twice the widths of the package's workloads, lengths are
theirs), `draw()` more of the same ranges.
"""
import math
import random

import torch

own = False

EPS = 1e-5          # of the normalisation (any small constant; the value does not change the work)


def listed():
    return [
        # One token for each of a few requests: the convolution's smallest call, nothing but latency.
        {"name": "conv_step_few", "op": "conv", "path": "step", "R": 4, "D": 1536, "m": 4, "dtype": "bf16"},
        # Prompts of different lengths, packed, some of them continued from the states of an earlier piece.
        {"name": "conv_prefill_packed", "op": "conv", "path": "fwd", "T": 6007, "seqs": 11, "D": 1536, "m": 4, "packed": True,
         "states": True, "dtype": "bf16"},
        # The convolution's share of a training step at the language-model width and length.
        {"name": "conv_train_lm", "op": "conv", "path": "train", "T": 65536, "seqs": 4, "D": 1536, "m": 4, "packed": False,
         "states": False, "dtype": "bf16"},
        # One token of one request: the scan's smallest call.
        {"name": "scan_step_one", "op": "scan", "path": "step", "R": 1, "D": 1536, "N": 16, "G": 1, "dtype": "bf16"},
        # A serving batch decoding together: every request's state is read and written once.
        {"name": "scan_step_batch", "op": "scan", "path": "step", "R": 256, "D": 1536, "N": 16, "G": 1, "dtype": "bf16"},
        # The packed prompts again, through the scan.
        {"name": "scan_prefill_packed", "op": "scan", "path": "fwd", "T": 6007, "seqs": 11, "D": 1536, "N": 16, "G": 1, "packed": True,
         "states": True, "dtype": "bf16"},
        # One prompt as long as the long-sequence workload's.
        {"name": "scan_prefill_long", "op": "scan", "path": "fwd", "T": 65536, "seqs": 1, "D": 2048, "N": 16, "G": 1, "packed": False,
         "states": True, "dtype": "bf16"},
        # Forward and backward at the language-model width and length: the largest case.
        {"name": "scan_train_lm", "op": "scan", "path": "train", "T": 65536, "seqs": 4, "D": 1536, "N": 16, "G": 1, "packed": False,
         "states": False, "dtype": "bf16"},
        # fp32, sequences of different lengths, grouped input and output maps, twice the state, a width that no tile divides.
        {"name": "scan_train_f32_packed", "op": "scan", "path": "train", "T": 3001, "seqs": 5, "D": 1000, "N": 32, "G": 2, "packed": True,
         "states": True, "dtype": "f32"},
        # The rows of a decoding batch.
        {"name": "norm_decode", "op": "norm", "path": "fwd", "T": 64, "D": 768, "dtype": "bf16"},
        # All rows of a training step at the language-model width.
        {"name": "norm_train_lm", "op": "norm", "path": "train", "T": 65536, "D": 768, "dtype": "bf16"},
        # fp32 rows of an odd width.
        {"name": "norm_train_f32_odd", "op": "norm", "path": "train", "T": 6007, "D": 1531, "dtype": "f32"},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case of the listed paths; lengths and widths are spread over their logarithm and mostly odd, and no case
    is larger than the largest listed one of its operator and path."""
    op = rng.choice(["conv", "scan", "scan", "norm"])
    dtype = "f32" if rng.random() < 0.3 else "bf16"
    D = rng.choice([512, 768, 1024, 1536, 2048]) if rng.random() < 0.6 else _log_int(rng, 100, 4096)
    if op == "norm":
        D = _log_int(rng, 100, 8192) if rng.random() < 0.4 else rng.choice([512, 768, 1024, 2048, 4096])
        return {"op": op, "path": rng.choice(["fwd", "train"]), "T": min(_log_int(rng, 1, 65536), 65536 * 768 // D), "D": D, "dtype": dtype}
    path = rng.choice(["step", "fwd", "train"])
    case = {"op": op, "path": path, "D": D, "dtype": dtype}
    if op == "conv":
        case["m"] = rng.choice([2, 3, 4, 4, 4, 5])
    else:
        case["N"] = rng.choice([8, 16, 16, 16, 32])
        case["G"] = rng.choice([1, 1, 1, 2, 4]) if D % 4 == 0 else 1
    if path == "step":
        case["R"] = min(_log_int(rng, 1, 512), max(1, 256 * 1536 * 16 // (D * case.get("N", 16))))
        return case
    most = 65536 * 1536 // (2 if dtype == "f32" else 1) * (16 if op == "scan" else 1)
    case["T"] = max(1, min(_log_int(rng, 16, 65536), most // (D * case.get("N", 1))))
    case["seqs"] = min(case["T"], _log_int(rng, 1, 32))
    case["packed"] = rng.random() < 0.5
    case["states"] = rng.random() < 0.5
    if not case["packed"]:
        case["T"] = case["T"] // case["seqs"] * case["seqs"]
    return case


def _lengths(case, seed):
    """The sequences' lengths: one each, or drawn with the seed (a sum of T, each at least one)."""
    if not case["packed"]:
        return [case["T"] // case["seqs"]] * case["seqs"]
    r = random.Random(int(seed) * 7919 + 1)
    cuts = sorted(r.sample(range(1, case["T"]), case["seqs"] - 1))
    return [b - a for a, b in zip([0] + cuts, cuts + [case["T"]])]


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))

    def randn(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    def rand(*shape):
        return torch.rand(*shape, generator=g, device="cuda")

    dt = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
    s, D, path = dict(case), case["D"], case["path"]
    if case["op"] == "norm":
        T = case["T"]
        # a residual stream that a few blocks have gone into, a silu gate, gains around one
        s.update(Y=randn(T, D).to(dt), X=(2 * randn(T, D)).to(dt), gate=torch.nn.functional.silu(randn(T, D)).to(dt),
                 w_post=1 + 0.1 * randn(D), w_pre=1 + 0.1 * randn(D), scale=0.5)
        if path == "train":
            s.update(dX_out=randn(T, D).to(dt), dN=randn(T, D).to(dt))
        return s
    step = path == "step"
    T = case["R"] if step else case["T"]
    n_seq = case["R"] if step else case["seqs"]
    if not step:
        s["lengths"] = _lengths(case, seed)
        s["max_len"] = max(s["lengths"])
        offsets = [0]
        for n in s["lengths"]:
            offsets.append(offsets[-1] + n)
        s["cu"] = torch.tensor(offsets, dtype=torch.int32, device="cuda")
        s["starts"] = torch.tensor(offsets[:-1], dtype=torch.int64, device="cuda")
        s["ends"] = torch.tensor(offsets[1:], dtype=torch.int64, device="cuda") - 1
        s["shape"] = (T, D) if case["packed"] else (n_seq, T // n_seq, D)
    states = step or case["states"]
    if case["op"] == "conv":
        m = case["m"]
        s.update(X=randn(T, D).to(dt), w=randn(D, m) / math.sqrt(m), bias=0.1 * randn(D))
        if states:
            s["S"] = randn(n_seq, m - 1, D).to(dt)
        if path == "train":
            s["dY"] = randn(T, D).to(dt)
            if states:
                s["dS_out"] = randn(n_seq, m - 1, D).to(dt)
        return s
    N, G = case["N"], case["G"]
    # step sizes of 1e-3 to 1e-1 after the softplus, decays of -1 to -N, as such layers are initialised; B and C are slices of the
    # projection that makes them
    size = torch.exp(rand(D) * math.log(100.0) + math.log(1e-3))
    both = randn(T, 2 * G * N).to(dt)
    s.update(U=torch.nn.functional.silu(randn(T, D)).to(dt), delta=(0.5 * randn(T, D)).to(dt), both=both,
             Bm=both[:, :G * N].unflatten(1, (G, N)), Cm=both[:, G * N:].unflatten(1, (G, N)),
             A=-(torch.arange(1, N + 1, device="cuda", dtype=torch.float32)[:, None] * torch.exp(0.1 * randn(N, D))),
             skip=1 + 0.1 * randn(D), Z=randn(T, D).to(dt), delta_bias=size + torch.log(-torch.expm1(-size)))
    if states:
        s["S"] = randn(n_seq, N, D)
    if path == "train":
        s["dY"] = randn(T, D).to(dt)
        if states:
            s["dS_out"] = randn(n_seq, N, D)
    return s


# ---- plain forms: elementary torch operations in 32 bits, rounded once at the end

def _silu(x):
    return x / (1 + torch.exp(-x))


def _dsilu(x):
    s = 1 / (1 + torch.exp(-x))
    return s * (1 + x * (1 - s))


def _position(s, T):
    """Of each row: its sequence, and its place in it."""
    row = torch.arange(T, device="cuda")
    seq = torch.searchsorted(s["ends"], row)
    return seq, row - s["starts"][seq]


def _taps(s, x, m, states):
    """[m, T, D]: x of t - j in t's sequence, from the state in front of it, or 0."""
    T, D = x.shape
    seq, place = _position(s, T)
    lag = place[None, :] - torch.arange(m, device="cuda")[:, None]
    row = s["starts"][seq][None, :] + lag
    got = torch.where((lag >= 0)[..., None], x[row.clamp(min=0)], x.new_zeros(()))
    if states is not None and m > 1:
        old = states.float()[seq[None, :].expand(m, T), (m - 1 + lag).clamp(0, m - 2)]
        got = torch.where((lag < 0)[..., None], old, got)
    return got


def _last_inputs(s, x, m, states):
    """[n_seq, m - 1, D]: the last m - 1 inputs of each sequence, those of the state among them where it is shorter."""
    length = s["ends"] - s["starts"] + 1
    place = length[:, None] + torch.arange(-(m - 1), 0, device="cuda")[None, :]
    new = x[(s["starts"][:, None] + place).clamp(min=0)]
    old = torch.gather(states, 1, (place + m - 1).clamp(0, m - 2)[..., None].expand_as(states))
    return torch.where((place >= 0)[..., None], new, old)


def _conv_plain(s):
    X, w, m, dt = s["X"].float(), s["w"], s["m"], s["X"].dtype
    if s["path"] == "step":
        x = torch.cat([s["S"].float(), X[:, None]], 1)
        y = _silu((x * w.t().flip(0)[None]).sum(1) + s["bias"])
        s["S"].copy_(x[:, 1:])
        return {"y": y.to(dt), "S": s["S"]}
    states = s.get("S")
    taps = _taps(s, X, m, states)
    u = (taps * w.t()[:, None, :]).sum(0) + s["bias"]
    out = {"Y": _silu(u).to(dt)}
    if states is not None:
        out["S_out"] = _last_inputs(s, s["X"], m, states)
    if s["path"] == "fwd":
        return out
    T, D = X.shape
    du = s["dY"].float() * _dsilu(u)
    out["dw"], out["dbias"] = (du[None] * taps).sum(1).t(), du.sum(0)
    seq, place = _position(s, T)
    length = (s["ends"] - s["starts"] + 1)
    lag = torch.arange(m, device="cuda")[:, None]
    ahead = torch.where(((place + lag) < length[seq])[..., None], du[(torch.arange(T, device="cuda") + lag).clamp(max=T - 1)], du.new_zeros(()))
    dX = (ahead * w.t()[:, None, :]).sum(0)
    if states is not None:
        # places -(m-1) .. -1 are the state in front of a sequence, and its last m - 1 places the one behind it
        dS_out = s["dS_out"].float()
        behind = place - (length[seq] - (m - 1))
        dX = dX + torch.where((behind >= 0)[:, None], dS_out[seq, behind.clamp(min=0)], dX.new_zeros(()))
        old = torch.arange(-(m - 1), 0, device="cuda")
        at = old[None, :, None] + torch.arange(m, device="cuda")[None, None, :]
        on = (at >= 0) & (at < length[:, None, None])
        rows = (s["starts"][:, None, None] + at).clamp(0, T - 1)
        dS = (torch.where(on[..., None], du[rows], du.new_zeros(())) * w.t()[None, None]).sum(2)
        behind = old[None, :] - (length[:, None] - (m - 1))
        dS = dS + torch.where((behind >= 0)[..., None], torch.gather(dS_out, 1, behind.clamp(min=0)[..., None].expand_as(dS_out)), dS.new_zeros(()))
        out["dS_in"] = dS.to(dt)
    out["dX"] = dX.to(dt)
    return out


def _running(a, b, length):
    """h_t = a_t h_{t-1} + b_t along the first dimension by doubling; a is 0 where a sequence begins, none is over `length`."""
    reach = 1
    while reach < length:
        b = torch.cat([b[:reach], torch.addcmul(b[reach:], a[reach:], b[:-reach])])
        a = torch.cat([a[:reach], a[reach:] * a[:-reach]])
        reach *= 2
    return b


def _spread(x, D):
    """[T, G, N] -> [T, N, D]: each group's row beside the channels that it serves."""
    T, G, N = x.shape
    return x.transpose(1, 2)[..., None].expand(T, N, G, D // G).reshape(T, N, D)


def _gather(x, G):
    """[T, N, D] -> [T, G, N]: the sum over each group's channels."""
    T, N, D = x.shape
    return x.reshape(T, N, G, D // G).sum(3).transpose(1, 2)


def _scan_plain(s):
    U, A, D, G, dt = s["U"].float(), s["A"], s["D"], s["G"], s["U"].dtype
    x = s["delta"].float() + s["delta_bias"]
    dl = torch.clamp(x, min=0) + torch.log1p(torch.exp(-x.abs()))
    Z = s["Z"].float()
    Bm, Cm = _spread(s["Bm"].float(), D), _spread(s["Cm"].float(), D)
    a = torch.exp(dl[:, None] * A)
    if s["path"] == "step":
        h = a * s["S"] + (dl * U)[:, None] * Bm
        y = ((Cm * h).sum(1) + s["skip"] * U) * _silu(Z)
        s["S"].copy_(h)
        return {"y": y.to(dt), "S": s["S"]}
    states = s.get("S")
    b = (dl * U)[:, None] * Bm
    if states is not None:
        b[s["starts"]] += a[s["starts"]] * states
    cut = a.clone()
    cut[s["starts"]] = 0
    h = _running(cut, b, s["max_len"])
    y = (Cm * h).sum(1) + s["skip"] * U
    out = {"Y": (y * _silu(Z)).to(dt)}
    if states is not None:
        out["S_out"] = h[s["ends"]]
    if s["path"] == "fwd":
        return out
    del b, cut
    dY = s["dY"].float()
    out["dZ"] = (dY * y * _dsilu(Z)).to(dt)
    dy = dY * _silu(Z)
    out["dskip"] = (dy * U).sum(0)
    out["dC"] = _gather(dy[:, None] * h, G).to(dt)
    # the gradient of a state is what its own output gives plus what the state behind it gives through that one's decay
    c = Cm * dy[:, None]
    if states is not None:
        c[s["ends"]] += s["dS_out"]
    behind = torch.cat([a[1:], torch.zeros_like(a[:1])])
    behind[s["ends"]] = 0
    g = _running(behind.flip(0), c.flip(0), s["max_len"]).flip(0)
    del c, behind
    if states is not None:
        out["dS_in"] = a[s["starts"]] * g[s["starts"]]
    out["dB"] = _gather(g * (dl * U)[:, None], G).to(dt)
    s1 = (g * Bm).sum(1)
    out["dU"] = (dl * s1 + s["skip"] * dy).to(dt)
    before = torch.cat([torch.zeros_like(h[:1]), h[:-1]])
    if states is not None:
        before[s["starts"]] = states
    else:
        before[s["starts"]] = 0
    before = g * a * before
    out["dA"] = (before * dl[:, None]).sum(0)
    dx = (U * s1 + (before * A).sum(1)) / (1 + torch.exp(-x))
    out["ddelta"], out["ddelta_bias"] = dx.to(dt), dx.sum(0)
    return out


def _norm_plain(s):
    Y, X, gate, dt = s["Y"].float(), s["X"].float(), s["gate"].float(), s["Y"].dtype
    r = 1 / torch.sqrt((Y * Y).mean(1, keepdim=True) + EPS)
    after = X + s["scale"] * (Y * r * s["w_post"] * gate)
    q = 1 / torch.sqrt((after * after).mean(1, keepdim=True) + EPS)
    out = {"X_out": after.to(dt), "N": (after * q * s["w_pre"]).to(dt)}
    if s["path"] == "fwd":
        return out
    # the backward pass has the stream as it was kept: rounded
    after = out["X_out"].float()
    q = 1 / torch.sqrt((after * after).mean(1, keepdim=True) + EPS)
    dN = s["dN"].float()
    out["dw_pre"] = (dN * after * q).sum(0)
    v, n = dN * s["w_pre"], after * q
    dX = s["dX_out"].float() + q * (v - n * (v * n).mean(1, keepdim=True))
    dp = s["scale"] * dX
    n = Y * r
    out["dgate"] = (dp * n * s["w_post"]).to(dt)
    out["dw_post"] = (dp * n * gate).sum(0)
    v = dp * s["w_post"] * gate
    out["dY"] = (r * (v - n * (v * n).mean(1, keepdim=True))).to(dt)
    out["dX"] = dX.to(dt)
    return out


# ---- the framework's calls

def _conv_own(s):
    from paper_2406_08128_amd import binding
    if s["path"] == "step":
        return {"y": binding.chela_short_conv_step(s["X"], s["w"], s["S"], bias=s["bias"]), "S": s["S"]}
    shape, cu = s["shape"], s["cu"] if s["packed"] else None
    X, S = s["X"].view(shape), s.get("S")
    S_out = torch.empty_like(S) if S is not None else None
    Y = binding.chela_short_conv_fwd(X, s["w"], bias=s["bias"], cu=cu, S_in=S, S_out=S_out)
    out = {"Y": Y.view(s["X"].shape)}
    if S is not None:
        out["S_out"] = S_out
    if s["path"] == "train":
        dX, dw, dbias, dS = binding.chela_short_conv_bwd(X, s["w"], s["dY"].view(shape), bias=s["bias"], cu=cu, S_in=S,
                                                         dS_out=s.get("dS_out"), want_dS_in=S is not None)
        out.update(dX=dX.view(s["X"].shape), dw=dw, dbias=dbias)
        if S is not None:
            out["dS_in"] = dS
    return out


def _scan_own(s):
    from paper_2406_08128_amd import binding
    if s["path"] == "step":
        y = binding.chela_selscan_step(s["U"], s["delta"], s["A"], s["Bm"], s["Cm"], s["S"], D=s["skip"], z=s["Z"], delta_bias=s["delta_bias"])
        return {"y": y, "S": s["S"]}
    shape, cu, S = s["shape"], s["cu"] if s["packed"] else None, s.get("S")
    U, delta, Z = (s[k].view(shape) for k in ("U", "delta", "Z"))
    Bm, Cm = (s[k].unflatten(0, shape[:-1]) if not s["packed"] else s[k] for k in ("Bm", "Cm"))
    kw = {"D": s["skip"], "Z": Z, "delta_bias": s["delta_bias"], "cu": cu, "S_in": S}
    S_out = torch.empty_like(S) if S is not None else None
    train = s["path"] == "train"
    Y, saved = binding.chela_selscan_fwd(U, delta, s["A"], Bm, Cm, S_out=S_out, want_saved=train, **kw)
    flat = s["U"].shape
    out = {"Y": Y.view(flat)}
    if S is not None:
        out["S_out"] = S_out
    if train:
        dU, ddelta, dA, dB, dC, dskip, dZ, dbias, dS = binding.chela_selscan_bwd(
            U, delta, s["A"], Bm, Cm, s["dY"].view(shape), dS_out=s.get("dS_out"), want_dS_in=S is not None, saved=saved, **kw)
        out.update(dU=dU.view(flat), ddelta=ddelta.view(flat), dA=dA, dB=dB.view(s["Bm"].shape), dC=dC.view(s["Cm"].shape), dskip=dskip,
                   dZ=dZ.view(flat), ddelta_bias=dbias)
        if S is not None:
            out["dS_in"] = dS
    return out


def _norm_own(s):
    from paper_2406_08128_amd import binding
    kw = {"gate": s["gate"], "w_post": s["w_post"], "w_pre": s["w_pre"], "scale": s["scale"], "eps": EPS}
    X_out, Nrm = binding.chela_block_norm_fwd(s["Y"], s["X"], **kw)
    out = {"X_out": X_out, "N": Nrm}
    if s["path"] == "train":
        dY, dgate, dX, dw_post, dw_pre = binding.chela_block_norm_bwd(s["Y"], X_out, s["dX_out"], s["dN"], **kw)
        out.update(dY=dY, dgate=dgate, dX=dX, dw_post=dw_post, dw_pre=dw_pre)
    return out


def run(s):
    if own:
        return {"conv": _conv_own, "scan": _scan_own, "norm": _norm_own}[s["op"]](s)
    return {"conv": _conv_plain, "scan": _scan_plain, "norm": _norm_plain}[s["op"]](s)


def work(case):
    es = 4 if case["dtype"] == "f32" else 2
    D, path = case["D"], case["path"]
    if case["op"] == "norm":
        e = case["T"] * D
        fwd = {"bytes": e * 5 * es + 8 * D, "flops": 10.0 * e}
        if path == "fwd":
            return fwd
        # Y gate X, dX_out dN; X_out N, dY dgate dX, and the gains' gradients
        return {"bytes": e * 10 * es + 16 * D, "flops": 40.0 * e}
    R = case["R"] if path == "step" else case["T"]
    seqs = R if path == "step" else case["seqs"] if case["states"] else 0
    e = R * D
    if case["op"] == "conv":
        m = case["m"]
        weights, state = (4 * m + 4) * D, seqs * (m - 1) * D * es
        if path != "train":
            return {"bytes": 2 * e * es + weights + 2 * state, "flops": e * (2.0 * m + 5)}
        return {"bytes": 4 * e * es + 2 * weights + 4 * state, "flops": e * (8.0 * m + 15)}
    N, G = case["N"], case["G"]
    weights, maps, state = (4 * N + 8) * D, 2 * R * G * N * es, seqs * N * D * 4
    if path != "train":
        return {"bytes": 4 * e * es + maps + weights + 2 * state, "flops": e * (7.0 * N + 20)}
    # U delta Z dY B C; Y dU ddelta dZ dB dC
    return {"bytes": 8 * e * es + 2 * maps + 2 * weights + 4 * state, "flops": e * (25.0 * N + 60)}


# ---- from the definition in 64 bits, one token after the other

def _by_sequence(x, s):
    """[T, ...] -> [n_seq, longest, ...], zeros behind the shorter ones."""
    out = x.new_zeros((len(s["lengths"]), s["max_len"]) + x.shape[1:])
    t = 0
    for i, n in enumerate(s["lengths"]):
        out[i, :n] = x[t:t + n]
        t += n
    return out


def _as_rows(x, s):
    return torch.cat([x[i, :n] for i, n in enumerate(s["lengths"])])


def _f64(s):
    return {k: v.double() if isinstance(v, torch.Tensor) and v.is_floating_point() else v for k, v in s.items()}


def _conv_exact(s):
    m, w, train, step = s["m"], s["w"], s["path"] == "train", s["path"] == "step"
    if step:
        s["lengths"], s["max_len"] = [1] * s["R"], 1
    leaves = [s["X"], w, s["bias"]] + ([s["S"]] if "S" in s else [])
    for t in leaves:
        t.requires_grad_(train)
    outs, keep, t0 = [], [], 0
    with torch.set_grad_enabled(train):
        for i, n in enumerate(s["lengths"]):
            front = s["S"][i] if "S" in s else s["X"].new_zeros(m - 1, s["D"])
            x = torch.cat([front, s["X"][t0:t0 + n]])
            u = s["bias"]
            for j in range(m):
                u = u + w[:, j] * x[m - 1 - j:m - 1 - j + n]
            outs.append(u * torch.sigmoid(u))
            keep.append(x[n:])
            t0 += n
        Y, S = torch.cat(outs), torch.stack(keep)
        if step:
            return {"y": Y, "S": S}
        got = {"Y": Y.detach()}
        if "S" in s:
            got["S_out"] = S.detach()
        if train:
            loss = (Y * s["dY"]).sum() + ((S * s["dS_out"]).sum() if "S" in s else 0)
            for k, v in zip(("dX", "dw", "dbias", "dS_in"), torch.autograd.grad(loss, leaves)):
                got[k] = v
    return got


def _scan_exact(s):
    D, N, G, step, train = s["D"], s["N"], s["G"], s["path"] == "step", s["path"] == "train"
    if step:
        s["lengths"], s["max_len"] = [1] * s["R"], 1
    raw = s["delta"] + s["delta_bias"]
    dl = torch.nn.functional.softplus(raw, threshold=700.0)
    gate = torch.sigmoid(s["Z"])
    per = D // G
    A = s["A"].reshape(N, G, per)
    # a step of size zero behind a sequence's end leaves its state as it is
    u, d = (_by_sequence(x, s).unflatten(2, (G, per)) for x in (s["U"], dl))
    Bm, Cm = (_by_sequence(x, s).transpose(2, 3) for x in (s["Bm"], s["Cm"]))          # [n, L, N, G]
    n, L = u.shape[:2]
    first = s["S"].reshape(n, N, G, per) if "S" in s else u.new_zeros(n, N, G, per)
    hs = u.new_empty(L, n, N, G, per) if train else None
    ys, h = u.new_empty(L, n, G, per), first
    for t in range(L):
        h = torch.exp(d[:, t, None] * A) * h + (d[:, t] * u[:, t])[:, None] * Bm[:, t, ..., None]
        ys[t] = (Cm[:, t, ..., None] * h).sum(1)
        if train:
            hs[t] = h
    y = _as_rows(ys.transpose(0, 1), s).reshape(-1, D) + s["skip"] * s["U"]
    Y, last = y * s["Z"] * gate, h.reshape(n, N, D)
    if step:
        return {"y": Y, "S": last}
    got = {"Y": Y}
    if "S" in s:
        got["S_out"] = last
    if not train:
        return got
    got["dZ"] = s["dY"] * y * (gate + s["Z"] * gate * (1 - gate))
    dy_rows = s["dY"] * s["Z"] * gate
    got["dskip"] = (dy_rows * s["U"]).sum(0)
    dy = _by_sequence(dy_rows, s).unflatten(2, (G, per))
    g = s["dS_out"].reshape(n, N, G, per) if "S" in s else torch.zeros_like(first)
    dB, dC = u.new_empty(L, n, G, N), u.new_empty(L, n, G, N)
    dd, dx, dA = u.new_empty(L, n, G, per), u.new_empty(L, n, G, per), torch.zeros_like(A)
    for t in range(L - 1, -1, -1):
        g = g + Cm[:, t, ..., None] * dy[:, t, None]
        dC[t] = (dy[:, t, None] * hs[t]).sum(3).transpose(1, 2)
        dB[t] = (g * (d[:, t] * u[:, t])[:, None]).sum(3).transpose(1, 2)
        into = (g * Bm[:, t, ..., None]).sum(1)
        dx[t] = d[:, t] * into
        g = torch.exp(d[:, t, None] * A) * g
        through = g * (hs[t - 1] if t else first)
        dA += (d[:, t, None] * through).sum(0)
        dd[t] = u[:, t] * into + (A * through).sum(1)
    if "S" in s:
        got["dS_in"] = g.reshape(n, N, D)
    got["dA"] = dA.reshape(N, D)
    got["dB"], got["dC"] = (_as_rows(x.transpose(0, 1), s) for x in (dB, dC))
    got["dU"] = _as_rows(dx.transpose(0, 1), s).reshape(-1, D) + s["skip"] * dy_rows
    draw_ = _as_rows(dd.transpose(0, 1), s).reshape(-1, D) * torch.sigmoid(raw)
    got["ddelta"], got["ddelta_bias"] = draw_, draw_.sum(0)
    return got


def _norm_exact(s, kept):
    def block(Y, X, gate, w_post):
        return X + s["scale"] * Y * (Y.square().mean(-1, keepdim=True) + EPS).rsqrt() * w_post * gate

    def norm(x, w):
        return x * (x.square().mean(-1, keepdim=True) + EPS).rsqrt() * w

    after = block(s["Y"], s["X"], s["gate"], s["w_post"])
    got = {"X_out": after, "N": norm(after, s["w_pre"])}
    if s["path"] == "fwd":
        return got
    with torch.enable_grad():
        x = after.to(kept).double().requires_grad_()
        w_pre = s["w_pre"].requires_grad_()
        dx, got["dw_pre"] = torch.autograd.grad((norm(x, w_pre) * s["dN"]).sum(), [x, w_pre])
        got["dX"] = dx + s["dX_out"]
        leaves = [s[k].requires_grad_() for k in ("Y", "gate", "w_post")]
        out = block(leaves[0], s["X"], leaves[1], leaves[2])
        got["dY"], got["dgate"], got["dw_post"] = torch.autograd.grad((out * got["dX"]).sum(), leaves)
    return got


def exact(case, seed):
    state = prepare(case, seed)
    kept = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
    s = _f64(state)
    if case["op"] == "norm":
        return {k: v.detach() for k, v in _norm_exact(s, kept).items()}
    with torch.no_grad():
        return (_conv_exact if case["op"] == "conv" else _scan_exact)(s)
