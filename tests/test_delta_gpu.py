"""The gated delta rule and the layer norm on the GPU against their definitions in 64 bits (oracle/delta.py).

Tolerances, before any run.
Element by element: half a step of the output's type, and what the roundings on the way may change, followed through the formulas of the chunks
(oracle.delta.delta_bounds: operands of matrix products rounded once, 2^-8, or held in two parts, 2^-16, for bf16; sums and exponentials in fp32).
That adds magnitudes up, so it says little where many terms cancel or decays are weak; therefore also
by norms, over a sequence and head: keys have length one and beta is at most one, so that no error of a state grows on its way, and the roundings are
independent of each other: the root of their number times half a step.  In bf16 an output has at most 8 on its way (state, inverse, inner values,
scores, twice for a gradient), 2^-8 sqrt(8); a state 6 of two parts, 2^-16 sqrt(6); in fp32 12 products of up to 128 terms, 2^-24 sqrt(12 128), which
may lie 4 times as high where a gradient adds several such terms of either sign; and half a step of the output's type on top.
Layer norm: mass (the same sums over magnitudes) times D + 64 roundings of 2^-24, rows on top for sums over rows."""
import numpy as np
import pytest
import torch

from oracle import delta as R
from oracle import rows as O
from paper_2406_08128_amd import binding

pytestmark = pytest.mark.gpu

HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
# Norms speak of many sums: a single token's gradient of its query is one sum of dv products times its key, and where those cancel by chance
# it is off by as much as it is itself, which only the bound element by element knows.
MANY = 16
BF, F32 = torch.bfloat16, torch.float32
DTYPES = [BF, F32]


def f64(t):
    return None if t is None else t.detach().double().cpu().numpy()


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return lambda *s: torch.randn(*s, generator=g, device="cuda")


def offsets(lens, first=0):
    return np.concatenate([[first], first + np.cumsum(lens)]).astype(np.int64)


def cu_of(lens, first=0):
    return torch.tensor(offsets(lens, first), dtype=torch.int32, device="cuda")


def wide_rows(t, lead, extra=3):
    """The same rows as a slice of wider ones, off 16-byte boundaries."""
    flat = t.reshape(*t.shape[:lead], -1)
    w = torch.full((*flat.shape[:-1], flat.shape[-1] + extra), float("nan"), dtype=t.dtype, device=t.device)
    w[..., 1:1 + flat.shape[-1]] = flat
    return w[..., 1:1 + flat.shape[-1]].unflatten(-1, t.shape[lead:])


def unit(x):
    return x / x.norm(dim=-1, keepdim=True)


def inputs(r, T, H, Hk, dk, dv, dtype, decay=2.0):
    """q, k of length one, v, g around -e^-decay, beta in (0, 1), dO."""
    return (unit(r(T, Hk, dk)).to(dtype), unit(r(T, Hk, dk)).to(dtype), r(T, H, dv).to(dtype), (-torch.exp(r(T, H) - decay)).to(dtype),
            torch.sigmoid(r(T, H)).to(dtype), r(T, H, dv).to(dtype))


def compare(what, got, ref, bound, state=False):
    half = HALF[got.dtype]
    g = f64(got)
    assert np.isfinite(g).all(), what
    if not ref.size:
        return
    off = np.abs(g - ref)
    tol = bound + half * (np.abs(ref) + bound) + 2.0 ** -126
    assert (off <= tol).all(), (what, float((off / tol).max()), np.unravel_index(int((off / tol).argmax()), off.shape))


def by_norm(what, got, ref, dtype, state=False, floor=0.0):
    half = HALF[got.dtype]
    rel = 2.0 ** -24 * 4 * np.sqrt(12 * 128)
    if dtype == BF:
        rel += 2.0 ** -16 * np.sqrt(6) if state else 2.0 ** -8 * np.sqrt(8)
    off = np.linalg.norm(f64(got) - ref)
    assert off <= (rel + half) * np.linalg.norm(ref) + np.linalg.norm(floor) + 1e-30, (what, off, np.linalg.norm(ref), rel + half)


def check_all(got, x, S, dS, lens, scale, dtype, first=0, bounds=True, skip=()):
    """Every output in `got` (by name, over all rows) against the definition, sequence by sequence and head by head."""
    q, k, v, g, beta, dO = (f64(t) for t in x)
    H, Hk = v.shape[1], k.shape[1]
    share, o = H // Hk, offsets(lens, first)
    chunk, once, twice = (64, 2.0 ** -8, 2.0 ** -16) if dtype == BF else (32, 0.0, 0.0)
    for i in range(len(lens)):
        a, b = o[i], o[i + 1]
        for hk in range(Hk):
            sums = {n: [0, 0] for n in ("dQ", "dK")}
            for h in range(hk * share, (hk + 1) * share):
                args = (q[a:b, hk], k[a:b, hk], v[a:b, h], None if g is None else g[a:b, h], beta[a:b, h])
                st, ds = None if S is None else f64(S[i, h]), None if dS is None else f64(dS[i, h])
                ref = dict(zip(("O", "S_out"), R.delta_fwd(*args, scale, st)))
                ref.update(R.delta_bwd(*args, dO[a:b, h], scale, st, ds))
                bound = R.delta_bounds(*args, dO[a:b, h], chunk, once, twice, scale, st, ds)
                for n in sums:
                    sums[n][0], sums[n][1] = sums[n][0] + ref[n], sums[n][1] + bound[n]
                for n in ("O", "S_out", "dV", "dg", "dbeta", "dS_in"):
                    if got.get(n) is None or (n, i) in skip:
                        continue
                    t = got[n][i, h] if n in ("S_out", "dS_in") else got[n][a:b, h]
                    if bounds:
                        compare((n, i, h), t, ref[n], bound[n])
                    if b - a >= MANY:
                        by_norm((n, i, h), t, ref[n], dtype, n in ("S_out", "dS_in"), bound["dg_sums"] if n == "dg" else 0.0)
            for n in sums:
                if got.get(n) is not None and b > a:
                    t = got[n][a:b, hk]
                    if bounds:
                        compare((n, i, hk), t, *sums[n])
                    if b - a >= MANY:
                        by_norm((n, i, hk), t, sums[n][0], dtype)


CASES = [  # H, Hk, dk, dv, lengths, states, gated, strided
    (1, 1, 64, 64, [1], True, True, False),
    (2, 2, 64, 64, [64], False, True, False),
    (2, 1, 64, 64, [5, 0, 63, 1, 65], True, True, False),
    (3, 1, 64, 128, [129, 17], True, True, True),
    (2, 2, 128, 64, [31, 33], True, False, True),
    (2, 1, 128, 128, [97, 2, 128], True, True, False),
    (4, 2, 64, 64, [32, 16, 15, 48], False, False, True),
]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("H,Hk,dk,dv,lens,states,gated,strided", CASES)
def test_gated_delta(dtype, H, Hk, dk, dv, lens, states, gated, strided):
    r, T, n = gen(H + dk + dv + len(lens)), sum(lens), len(lens)
    q, k, v, g, beta, dO = inputs(r, T, H, Hk, dk, dv, dtype)
    g = g if gated else None
    S, dS = (0.3 * r(n, H, dk, dv), 0.3 * r(n, H, dk, dv)) if states else (None, None)
    x = [wide_rows(t, 1) if strided and t is not None else t for t in (q, k, v, g, beta, dO)]
    kw = dict(scale=0.125, cu=cu_of(lens), S_in=S)
    S_out = torch.full((n, H, dk, dv), float("nan"), device="cuda")
    out, saved = binding.chela_gated_delta_fwd(*x[:5], S_out=S_out, want_saved=True, **kw)
    grads = binding.chela_gated_delta_bwd(*x[:5], x[5], dS_out=dS, want_dS_in=True, saved=saved, **kw)
    again = binding.chela_gated_delta_bwd(*x[:5], x[5], dS_out=dS, want_dS_in=True, **kw)
    for a, b in zip(grads, again):
        assert (a is None) == (b is None) and (a is None or torch.equal(a, b))
    assert (grads[3] is None) == (not gated)
    got = dict(zip(("dQ", "dK", "dV", "dg", "dbeta", "dS_in"), grads), O=out, S_out=S_out)
    check_all(got, (q, k, v, g, beta, dO), S, dS, lens, 0.125, dtype)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("dk,dv", [(64, 64), (128, 128)])
def test_many_chunks(dtype, dk, dv):
    # long enough for a state to go through many of them, decays that keep it and decays that do not
    r, H, L = gen(dk), 2, 700
    x = inputs(r, 2 * L, H, 1, dk, dv, dtype, decay=4.0)
    S, dS = 0.3 * r(2, H, dk, dv), 0.3 * r(2, H, dk, dv)
    v3 = [t.view(2, L, *t.shape[1:]) for t in x]
    S_out = torch.empty_like(S)
    out, saved = binding.chela_gated_delta_fwd(*v3[:5], scale=0.1, S_in=S, S_out=S_out, want_saved=True)
    grads = binding.chela_gated_delta_bwd(*v3[:5], v3[5], scale=0.1, S_in=S, dS_out=dS, want_dS_in=True, saved=saved)
    got = {n: t.flatten(0, 1) for n, t in zip(("dQ", "dK", "dV", "dg", "dbeta"), grads)}
    check_all(dict(got, O=out.flatten(0, 1), S_out=S_out, dS_in=grads[5]), x, S, dS, [L, L], 0.1, dtype, bounds=False)


RUNS = [  # lengths long enough for runs of several chunks; sequences whose last run is short or ends inside a chunk, that have less than one run
    (1, 1, 64, 64, [1100]),
    (2, 2, 64, 128, [1400, 3]),
    (2, 1, 128, 64, [577, 1090, 0, 1029]),
    (1, 1, 128, 128, [2305]),
    (2, 2, 64, 64, [4200, 5]),
    (2, 2, 128, 64, [1100, 577]),
    (1, 1, 64, 128, [8300]),
]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("states", [False, True])
@pytest.mark.parametrize("H,Hk,dk,dv,lens", RUNS)
def test_runs_of_chunks(dtype, states, H, Hk, dk, dv, lens):
    # nothing kept, kept for a gradient, a gradient that has nothing kept; decays that keep a state over many chunks
    r, T, n = gen(dk + dv + len(lens)), sum(lens), len(lens)
    x = inputs(r, T, H, Hk, dk, dv, dtype, decay=5.0)
    S, dS = (0.3 * r(n, H, dk, dv), 0.3 * r(n, H, dk, dv)) if states else (None, None)
    kw = dict(scale=0.1, cu=cu_of(lens), S_in=S)
    S_out = torch.empty(n, H, dk, dv, device="cuda") if states else None
    O0, _ = binding.chela_gated_delta_fwd(*x[:5], S_out=S_out, **kw)
    check_all(dict(O=O0, S_out=S_out), x, S, dS, lens, 0.1, dtype, bounds=False)
    O1, saved = binding.chela_gated_delta_fwd(*x[:5], S_out=S_out, want_saved=True, **kw)
    grads = binding.chela_gated_delta_bwd(*x[:5], x[5], dS_out=dS, want_dS_in=states, saved=saved, **kw)
    again = binding.chela_gated_delta_bwd(*x[:5], x[5], dS_out=dS, want_dS_in=states, **kw)
    names = ("dQ", "dK", "dV", "dg", "dbeta", "dS_in")
    check_all(dict(zip(names, grads), O=O1, S_out=S_out), x, S, dS, lens, 0.1, dtype, bounds=False)
    check_all(dict(zip(names, again)), x, S, dS, lens, 0.1, dtype, bounds=False)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("lens", [[1] * 10, [1100, 3, 0, 64, 1]])
def test_a_first_token_lets_nothing_decay(dtype, lens):
    r, T, H = gen(8), sum(lens), 2
    x = inputs(r, T, H, H, 64, 64, dtype)
    dg = binding.chela_gated_delta_bwd(*x, cu=cu_of(lens))[3]
    starts = torch.tensor([a for a, n in zip(offsets(lens), lens) if n], device="cuda")
    assert (dg[starts] == 0).all() and (T == len(starts) or (dg != 0).sum() >= (T - len(starts)) * H // 2)


@pytest.mark.parametrize("dtype", DTYPES)
def test_in_place_states_pieces_and_single_tokens(dtype):
    r, H, Hk, dk, dv, n, L = gen(5), 4, 2, 64, 64, 3, 150
    x = inputs(r, n * L, H, Hk, dk, dv, dtype)
    v3 = [t.view(n, L, *t.shape[1:]) for t in x[:5]]
    S = 0.3 * r(n, H, dk, dv)
    S2, S_out = S.clone(), torch.empty_like(S)
    a, _ = binding.chela_gated_delta_fwd(*v3, S_in=S, S_out=S_out)
    b, _ = binding.chela_gated_delta_fwd(*v3, S_in=S2, S_out=S2)
    c, _ = binding.chela_gated_delta_fwd(*x[:5], cu=cu_of([L] * n), S_in=S)
    assert torch.equal(a, b) and torch.equal(S_out, S2) and torch.equal(a.flatten(0, 1), c)
    S3, got, t = S.clone(), [], 0
    for m in (1, 70, 65):
        got.append(binding.chela_gated_delta_fwd(*(y[:, t:t + m].contiguous() for y in v3), S_in=S3, S_out=S3)[0])
        t += m
    for t in range(t, L):
        got.append(binding.chela_gated_delta_step(*(y[:, t] for y in v3), S3)[:, None])        # (rows with a stride)
    check_all(dict(O=torch.cat(got, 1).flatten(0, 1), S_out=S3), x, S, None, [L] * n, 1.0, dtype)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("H,Hk,dk,dv,gated", [(1, 1, 64, 64, True), (6, 2, 64, 128, True), (3, 3, 128, 64, False), (2, 1, 128, 128, True)])
def test_step_against_the_definition(dtype, H, Hk, dk, dv, gated):
    r, n = gen(dk + dv + H), 5
    q, k, v, g, beta, _ = inputs(r, n, H, Hk, dk, dv, dtype)
    g = g if gated else None
    S = r(n, H, dk, dv)
    for strided in (False, True):
        S2 = S.clone()
        x = [wide_rows(t, 1) if strided and t is not None else t for t in (q, k, v, g, beta)]
        o = binding.chela_gated_delta_step(*x, S2, scale=0.3)
        for i in range(n):
            for h in range(H):
                hk = h // (H // Hk)
                args = (f64(q[i:i + 1, hk]), f64(k[i:i + 1, hk]), f64(v[i:i + 1, h]), f64(g[i:i + 1, h]) if gated else None, f64(beta[i:i + 1, h]))
                ref, after = R.delta_fwd(*args, 0.3, f64(S[i, h]))
                a = np.exp(args[3][0]) if gated else 1.0
                # dk terms of either product, and a few roundings more
                read = np.abs(args[2][0]) + a * np.abs(args[1][0]) @ np.abs(f64(S[i, h]))
                ms = a * np.abs(f64(S[i, h])) + np.outer(np.abs(args[1][0]), args[4][0] * read)
                compare("S", S2[i, h], after, (dk + 16) * R.F * ms)
                compare("o", o[i, h], ref[0], 0.3 * (2 * dk + 32) * R.F * (np.abs(args[0][0]) @ ms))


@pytest.mark.parametrize("dtype", DTYPES)
def test_slots_and_rows_of_nobody(dtype):
    r, H, Hk, dk, dv = gen(17), 2, 1, 64, 64
    lens, first, T = [5, 0, 70, 1, 90], 3, 180                     # rows 0 .. 2 and 169 .. 179 are nobody's
    cu, n, o = cu_of(lens, first), len(lens), offsets(lens, first)
    slots = torch.tensor([6, 2, -1, 0, 99], dtype=torch.int32, device="cuda")        # a pool of 8; sequences 2 and 4 have no state
    x = inputs(r, T, H, Hk, dk, dv, dtype)
    owned = torch.zeros(T, dtype=torch.bool, device="cuda")
    owned[o[0]:o[-1]] = True
    for t in x:
        t[~owned] = float("nan")                                   # nothing of these rows is taken in
    mark = 12345.0
    pool = 0.3 * r(8, H, dk, dv)
    p0 = pool.clone()
    out = torch.full((T, H, dv), mark, dtype=dtype, device="cuda")
    binding.chela_gated_delta_fwd(*x[:5], cu=cu, S_in=pool, S_out=pool, slots=slots, O=out)
    assert (out[~owned] == out.new_tensor(mark)).all()
    where = {0: 6, 1: 2, 3: 0}
    S = torch.zeros(n, H, dk, dv, device="cuda")
    S_out = torch.zeros_like(S)
    for i, s in where.items():
        S[i], S_out[i] = p0[s], pool[s]
    check_all(dict(O=out, S_out=S_out), x, S, None, lens, 1.0, dtype, first, skip={("S_out", 2), ("S_out", 4)})
    for s in range(8):
        if s not in where.values():
            assert torch.equal(pool[s], p0[s])
    new, _ = binding.chela_gated_delta_fwd(*x[:5], cu=cu, S_in=p0, slots=slots)
    assert (new[~owned] == 0).all() and torch.equal(new[owned], out[owned])
    grads = binding.chela_gated_delta_bwd(*x[:5], x[5], cu=cu, want_dS_in=True)
    for t in grads[:5]:
        assert (t[~owned] == 0).all() and torch.isfinite(t.float()).all()
    zero = binding.chela_gated_delta_fwd(*x[:5], cu=cu)[0]
    check_all(dict(zip(("dQ", "dK", "dV", "dg", "dbeta", "dS_in"), grads), O=zero), x, None, None, lens, 1.0, dtype, first)
    # single tokens: rows without a slot stay, or are zero in a new tensor
    y = torch.full((n, H, dv), mark, dtype=dtype, device="cuda")
    tok = [t[owned][:n].contiguous() for t in x[:5]]
    before = pool.clone()
    binding.chela_gated_delta_step(*tok, pool, slots=slots, o=y)
    z = binding.chela_gated_delta_step(*tok, before.clone(), slots=slots)
    for i in range(n):
        if i in where:
            assert not torch.equal(pool[where[i]], before[where[i]]) and (y[i] != y.new_tensor(mark)).any() and torch.equal(y[i], z[i])
        else:
            assert (y[i] == y.new_tensor(mark)).all() and (z[i] == 0).all()
    for s in range(8):
        if s not in where.values():
            assert torch.equal(pool[s], before[s])


@pytest.mark.parametrize("n", [70, 5000])
def test_many_sequences(n):
    # more than one, and more than 64 times 64, to look through for a chunk's
    r, H, dk, dv = gen(n), 1, 64, 64
    lens = [(7 * i) % 5 if i % 50 else 66 for i in range(n)]
    T = sum(lens)
    x = inputs(r, T, H, 1, dk, dv, F32)
    S = 0.3 * r(n, H, dk, dv)
    S_out = torch.full_like(S, float("nan"))
    out, _ = binding.chela_gated_delta_fwd(*x[:5], cu=cu_of(lens), S_in=S, S_out=S_out)
    grads = binding.chela_gated_delta_bwd(*x[:5], x[5], cu=cu_of(lens), S_in=S)
    o = offsets(lens)
    for i in list(range(0, n, 50)) + [1, 63, 64, 65, n - 2, n - 1]:
        a, b = o[i], o[i + 1]
        one = tuple(t[a:b] for t in x)
        got = dict({m: t[a:b] for m, t in zip(("dQ", "dK", "dV", "dg", "dbeta"), grads)}, O=out[a:b], S_out=S_out[i:i + 1])
        check_all(got, one, S[i:i + 1], None, [lens[i]], 1.0, F32)
    empty = torch.tensor([m == 0 for m in lens], device="cuda")
    assert torch.equal(S_out[empty], S[empty])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("cu", [[0, 900, 300, 1200, 700, 1500], [1500, 0, 1500, 0], [-70, 400, 399, 2000, 2000, 0, 1 << 30]])
def test_offsets_out_of_order_stay_inside(dtype, cu):
    # what they give is not specified; nothing in front of or behind the tensors is touched, and calls behind these are right
    r, T, H, n, pad = gen(3), 1500, 2, len(cu) - 1, 4096
    x = inputs(r, T, H, H, 64, 64, dtype)
    cu = torch.tensor(cu, dtype=torch.int32, device="cuda")
    S = 0.1 * r(n, H, 64, 64)
    room = torch.full((T * H * 64 + 2 * pad,), 7.0, dtype=dtype, device="cuda")
    O = room[pad:-pad].view(T, H, 64)
    for states in (False, True):
        kw = dict(cu=cu, S_in=S if states else None)
        _, saved = binding.chela_gated_delta_fwd(*x[:5], S_out=torch.empty_like(S) if states else None, want_saved=True, O=O, **kw)
        binding.chela_gated_delta_fwd(*x[:5], O=O, **kw)
        binding.chela_gated_delta_bwd(*x, saved=saved, **kw)
        binding.chela_gated_delta_bwd(*x, **kw)
    assert (room[:pad] == 7).all() and (room[-pad:] == 7).all()
    out, _ = binding.chela_gated_delta_fwd(*x[:5], cu=cu_of([T]))
    check_all(dict(O=out), x, None, None, [T], 1.0, dtype, bounds=False)


@pytest.mark.parametrize("dtype", DTYPES)
def test_no_rows_and_no_sequences(dtype):
    H, dk, dv = 2, 64, 128
    e = lambda *s: torch.empty(*s, dtype=dtype, device="cuda")  # noqa: E731
    S = gen(3)(3, H, dk, dv)
    S_out = torch.full_like(S, float("nan"))
    x = (e(0, H, dk), e(0, H, dk), e(0, H, dv), e(0, H), e(0, H))
    cu = torch.zeros(4, dtype=torch.int32, device="cuda")
    out, saved = binding.chela_gated_delta_fwd(*x, cu=cu, S_in=S, S_out=S_out, want_saved=True)
    assert out.shape == (0, H, dv) and torch.equal(S_out, S)
    g = binding.chela_gated_delta_bwd(*x, e(0, H, dv), cu=cu, S_in=S, dS_out=S, want_dS_in=True, saved=saved)
    assert torch.equal(g[5], S)
    S_out.fill_(float("nan"))
    x3 = tuple(t.view(3, 0, *t.shape[1:]) for t in x)
    binding.chela_gated_delta_fwd(*x3, S_in=S, S_out=S_out)
    assert torch.equal(S_out, S)
    # rows, and no sequence that has them
    x = inputs(gen(4), 70, H, H, dk, dv, dtype)
    none = torch.zeros(1, dtype=torch.int32, device="cuda")
    out, _ = binding.chela_gated_delta_fwd(*x[:5], cu=none)
    assert (out == 0).all()
    assert all((t == 0).all() for t in binding.chela_gated_delta_bwd(*x[:5], x[5], cu=none)[:5])
    assert binding.chela_gated_delta_step(*(t[:0] for t in x[:5]), S[:0]).shape == (0, H, dv)


@pytest.mark.parametrize("dtype", DTYPES)
def test_extreme_decays_and_strengths(dtype):
    r, H, dk, dv, L = gen(23), 6, 64, 64, 140
    q, k, v, g, beta, dO = inputs(r, L, H, H, dk, dv, dtype)
    g[:, 0] = 0                                            # nothing decays
    g[:, 1] = -float("inf")                                # nothing is left of a token
    g[:, 2] = torch.where(torch.arange(L, device="cuda") % 9 == 0, -float("inf"), g[:, 2].float()).to(dtype)
    g[:, 3] = -90.0
    g[:, 4] = torch.where(torch.arange(L, device="cuda") % 40 == 5, torch.finfo(dtype).min, 0.0).to(dtype)     # sequences in a row, as a mask makes them
    beta[:, 0], beta[:, 1] = 1, 0
    beta[::3, 2] = 0
    beta[:, 5] = 1
    k[:, 5] = k[0, 5]                                      # one key for all tokens: each replaces what the one in front wrote
    S, dS = r(1, H, dk, dv), r(1, H, dk, dv)
    S_out = torch.empty_like(S)
    x = (q, k, v, g, beta, dO)
    v3 = [t[None] for t in x]
    out, saved = binding.chela_gated_delta_fwd(*v3[:5], S_in=S, S_out=S_out, want_saved=True)
    grads = binding.chela_gated_delta_bwd(*v3[:5], v3[5], S_in=S, dS_out=dS, want_dS_in=True, saved=saved)
    for t in (out, S_out, *grads):
        assert torch.isfinite(t).all()
    got = {n: t[0] for n, t in zip(("dQ", "dK", "dV", "dbeta"), (*grads[:3], grads[4]))}
    g64 = tuple(t if i != 3 else t.clamp(min=-1e4) for i, t in enumerate(x))
    # (head 5's rows cancel each other: magnitudes say what is left of them, norms do not)
    heads = [slice(0, 5)]
    for s in heads:
        check_all({n: t[:, s] for n, t in got.items()} | dict(O=out[0][:, s], S_out=S_out[:, s], dS_in=grads[5][:, s]),
                  tuple(t[:, s] for t in g64), S[:, s], dS[:, s], [L], 1.0, dtype, bounds=False)
    assert torch.equal(S_out[0, 1], torch.zeros_like(S_out[0, 1])) and torch.equal(grads[5][0, 1], torch.zeros_like(S_out[0, 1]))
    # one key, beta of one, no decay to speak of: what is read at the key is the last value
    read = (k[0, 5].float() @ S_out[0, 5])
    assert (read - v[-1, 5].float()).norm() <= 0.02 * v[-1, 5].float().norm()


@pytest.mark.parametrize("dtype", DTYPES)
def test_what_is_not_finite_stays_in_its_sequence(dtype):
    r, H, dk, dv = gen(29), 2, 64, 64
    lens = [70, 20, 90]
    x = inputs(r, 180, H, H, dk, dv, dtype)
    bad = [t.clone() for t in x]
    o = offsets(lens)
    for t, val in zip(bad, (float("nan"), float("inf"), float("nan"), float("nan"), float("inf"), float("nan"))):
        t[o[1]:o[2]] = val
    a = binding.chela_gated_delta_fwd(*x[:5], cu=cu_of(lens), want_saved=True)
    b = binding.chela_gated_delta_fwd(*bad[:5], cu=cu_of(lens), want_saved=True)
    ga = binding.chela_gated_delta_bwd(*x[:5], x[5], cu=cu_of(lens), saved=a[1])
    gb = binding.chela_gated_delta_bwd(*bad[:5], bad[5], cu=cu_of(lens), saved=b[1])
    keep = torch.ones(180, dtype=torch.bool, device="cuda")
    keep[o[1]:o[2]] = False
    for p, q in zip((a[0], *ga[:5]), (b[0], *gb[:5])):
        assert torch.equal(p[keep], q[keep])
    # a token's value reaches none in front of its chunk
    y = [t.clone() for t in x]
    y[2][150] = float("nan")
    c = binding.chela_gated_delta_fwd(*y[:5], cu=cu_of(lens))[0]
    front = 90 + (60 // (64 if dtype == BF else 32)) * (64 if dtype == BF else 32)
    assert torch.equal(c[:front], a[0][:front]) and not torch.isfinite(c[150:]).any()


@pytest.mark.parametrize("dtype", DTYPES)
def test_what_is_not_finite_stays_on_its_side_of_its_chunk(dtype):
    # in runs of several chunks too: values reach no chunk in front, upstream gradients none behind
    C, T, H = 64 if dtype == BF else 32, 1400, 2
    x = inputs(gen(31), T, H, H, 64, 64, dtype)
    y = [t.clone() for t in x]
    y[2][1000], y[1][1003], y[4][1001] = float("nan"), float("inf"), float("nan")
    for kept in (False, True):
        a, b = (binding.chela_gated_delta_fwd(*t[:5], want_saved=kept) for t in (x, y))
        front = 1000 // C * C
        assert torch.equal(a[0][:front], b[0][:front]) and not torch.isfinite(b[0][1003:]).any()
    z = [t.clone() for t in x]
    z[5][500] = float("nan")
    behind = (500 // C + 1) * C
    for p, q in zip(binding.chela_gated_delta_bwd(*x)[:5], binding.chela_gated_delta_bwd(*z)[:5]):
        assert torch.equal(p[behind:], q[behind:])


# ------------------------------------------------------------------------------------------- layer norm
def check(name, got, ref, mass, n):
    tol = O.tolerance(ref, mass, n, HALF[got.dtype])
    off = np.abs(f64(got) - ref)
    assert np.isfinite(f64(got)).all(), name
    worst = float((off / tol).max()) if off.size else 0.0
    assert worst <= 1.0, (name, worst)


NORM = [(1, 1), (3, 2), (4, 5), (7, 64), (5, 255), (33, 768), (9, 1000), (600, 513), (6, 1025), (5, 2047), (4, 4096), (3, 4097), (3, 8191), (2, 8192)]


@pytest.mark.parametrize("dtype,x_f32", [(BF, False), (BF, True), (F32, False)])
@pytest.mark.parametrize("rows,D", NORM)
def test_layer_norm(dtype, x_f32, rows, D):
    r = gen(rows + D)
    xt = F32 if x_f32 else dtype
    X, Y, w, b = (2 * r(rows, D) + 3).to(xt), r(rows, D).to(dtype), 1 + 0.3 * r(D), r(D)
    dN, dX_out = r(rows, D).to(dtype), r(rows, D).to(xt)
    for w_, b_, y_, up in ((w, b, Y, dX_out), (w, None, Y, None), (None, b, Y, dX_out), (None, None, None, None), (w, b, None, dX_out)):
        if y_ is None and x_f32:
            N = torch.empty(rows, D, dtype=dtype, device="cuda")
            after, N = binding.chela_layer_norm_fwd(X, w=w_, b=b_, Nrm=N)
        else:
            after, N = binding.chela_layer_norm_fwd(X, w=w_, b=b_, Y=y_)
        assert (after is X) == (y_ is None)
        v, m = R.layer_norm_fwd(f64(X), f64(y_), f64(w_), f64(b_))
        check("X_out", after, v["X_out"], m["X_out"], 2)
        check("N", N, v["N"], m["N"], D + 64)
        g = binding.chela_layer_norm_bwd(after, dN, w=w_, want_db=b_ is not None, dX_out=up)
        v, m = R.layer_norm_bwd(f64(after), f64(dN), f64(w_), f64(up))
        check("dX", g[0], v["dX"], m["dX"], D + 64)
        assert (g[1] is None) == (w_ is None) and (g[2] is None) == (b_ is None)
        if w_ is not None:
            check("dw", g[1], v["dw"], m["dw"], D + rows + 64)
        if b_ is not None:
            check("db", g[2], v["db"], m["db"], rows + 64)


def test_layer_norm_in_place_and_far_from_zero():
    r, D = gen(3), 768
    X, Y, w = r(50, D).to(BF), r(50, D).to(BF), 1 + 0.1 * r(D)
    a = binding.chela_layer_norm_fwd(X, w=w, Y=Y)
    x = X.clone()
    b = binding.chela_layer_norm_fwd(x, w=w, Y=Y, X_out=x)
    assert b[0] is x and torch.equal(a[0], x) and torch.equal(a[1], b[1])
    x = X.clone()
    c = binding.chela_layer_norm_fwd(x, w=w, Y=x, X_out=x)                 # the same tensor twice
    d = binding.chela_layer_norm_fwd(X, w=w, Y=X.clone())
    assert torch.equal(c[0], d[0]) and torch.equal(c[1], d[1])
    dN, up = r(50, D).to(BF), r(50, D).to(BF)
    g = binding.chela_layer_norm_bwd(a[0], dN, w=w, dX_out=up)
    u = up.clone()
    h = binding.chela_layer_norm_bwd(a[0], dN, w=w, dX_out=u, in_place=True)
    assert h[0] is u and torch.equal(g[0], u) and torch.equal(g[1], h[1])
    u = up.clone()
    e = binding.chela_layer_norm_bwd(a[0], u, w=w, dX_out=u, in_place=True)         # one upstream gradient for both
    f = binding.chela_layer_norm_bwd(a[0], up, w=w, dX_out=up.clone())
    assert torch.equal(e[0], f[0]) and torch.equal(e[1], f[1])
    # rows that are 1000 everywhere but for a little: the squares are of the little
    X = 1000 + 0.01 * r(20, D)
    N = binding.chela_layer_norm_fwd(X, eps=0.0)[1]
    x = f64(X)
    c = x - x.mean(1, keepdims=True)
    # the mean's own roundings, D of them on 1000, go off every element alike: they move n by that over the rows' size, and its square the size
    off = D * 2.0 ** -24 * 1000 / np.sqrt((c ** 2).mean(1, keepdims=True))
    n = c / np.sqrt((c ** 2).mean(1, keepdims=True))
    assert (np.abs(f64(N) - n) <= off * (1 + np.abs(n)) + (D + 64) * 2.0 ** -24 * np.abs(n)).all()
    # and rows that are the same everywhere
    N = binding.chela_layer_norm_fwd(torch.full((3, D), 5.0, device="cuda"), b=w)[1]
    assert torch.allclose(N, w.expand(3, D), atol=1e-6)
    out = binding.chela_layer_norm_bwd(torch.empty(0, D, device="cuda"), torch.empty(0, D, device="cuda"), w=w, want_db=True)
    assert out[0].shape == (0, D) and (out[1] == 0).all() and (out[2] == 0).all()
    assert binding.chela_layer_norm_fwd(torch.empty(0, D, device="cuda"), w=w)[1].shape == (0, D)


# ------------------------------------------------------------------------------------------- together
def _block(D, H, Hk, dk, m, r):
    """A block as a model has it: layer norm with the residual, projections, short convolution, rows of length one, delta rule, gated norm."""
    wide = 2 * Hk * dk + H * dk
    p = dict(w=1 + 0.1 * r(D), b=0.1 * r(D), proj=(r(D, wide) / D ** 0.5).to(BF), gates=(r(D, 2 * H) / D ** 0.5).to(BF), conv=0.5 * r(wide, m),
             unit=torch.full((dk,), dk ** -0.5, device="cuda"), gate=(r(D, H * dk) / D ** 0.5).to(BF), out=(r(H * dk, D) / (H * dk) ** 0.5).to(BF))

    def mm(x, w):                                     # (row by row the same sums, up to their order)
        return (x.float().reshape(-1, x.shape[-1]) @ w.float()).to(BF).view(*x.shape[:-1], w.shape[1])

    def run(X, Y, conv, rule):
        X, h = binding.chela_layer_norm_fwd(X, w=p["w"], b=p["b"], Y=Y)
        qkv = conv(mm(h, p["proj"]), p["conv"])
        lead = qkv.shape[:-1]
        q, k, v = (t.unflatten(-1, (-1, dk)) for t in qkv.split([Hk * dk, Hk * dk, H * dk], -1))
        q, k = (binding.chela_block_norm_fwd(None, t.contiguous(), w_pre=p["unit"])[1] for t in (q, k))
        a = mm(h, p["gates"])
        g, beta = -torch.nn.functional.softplus(a[..., :H].float()).to(BF), torch.sigmoid(a[..., H:].float()).to(BF)
        o = rule(q, k, v, g, beta)
        y = binding.chela_gate_norm_fwd(o.reshape(1, 1, -1, dk), torch.nn.functional.silu(mm(h, p["gate"]).float()).to(BF).reshape(1, 1, -1, dk), 1e-5)
        return X, mm(y.reshape(*lead, H * dk), p["out"])

    return run


def test_a_block_prompt_then_tokens_is_the_sequence():
    r, n, L, D, H, Hk, dk, m, cut = gen(31), 2, 100, 128, 2, 1, 64, 4, 83
    run = _block(D, H, Hk, dk, m, r)
    wide = 2 * Hk * dk + H * dk
    X, Y = r(n, L, D).to(BF), r(n, L, D).to(BF)

    def whole(x, y, C, S):
        return run(x, y, lambda t, w: binding.chela_short_conv_fwd(t, w, S_in=C, S_out=C),
                   lambda *a: binding.chela_gated_delta_fwd(*a, scale=dk ** -0.5, S_in=S, S_out=S)[0])

    def token(x, y, C, S):
        return run(x, y, lambda t, w: binding.chela_short_conv_step(t, w, C), lambda *a: binding.chela_gated_delta_step(*a, S, scale=dk ** -0.5))

    def fresh():
        return torch.zeros(n, m - 1, wide, dtype=BF, device="cuda"), torch.zeros(n, H, dk, dk, device="cuda")

    C, S = fresh()
    one = whole(X, Y, C, S)
    C2, S2 = fresh()
    parts = [whole(X[:, :cut].contiguous(), Y[:, :cut].contiguous(), C2, S2)]
    parts += [tuple(t[:, None] for t in token(X[:, t].contiguous(), Y[:, t].contiguous(), C2, S2)) for t in range(cut, L)]
    # every stage rounds to bf16, and sums taken in another order, or rounded as operands, may round the other way: the rule's own 8 roundings
    # and those of the five stages around it, each a step of the largest values
    for i in range(2):
        got = torch.cat([p[i] for p in parts], 1).float()
        assert (got - one[i].float()).abs().max() <= 13 * 2.0 ** -8 * one[i].float().abs().max()
    assert (S - S2).abs().max() <= 8 * 2.0 ** -8 * S.abs().max()


# ------------------------------------------------------------------------------------------- streams, graphs, threads, sizes
def _training_pass(T, H, Hk, dk, dv, dtype, seed):
    r = gen(seed)
    x = inputs(r, T, H, Hk, dk, dv, dtype)
    q, k, v, g, beta, dO = x
    w, b = 1 + 0.1 * r(H * dv), 0.1 * r(H * dv)
    cu = cu_of([T // 3, 0, T - T // 3])
    S = 0.3 * r(3, H, dk, dv)

    def run():
        X, h = binding.chela_layer_norm_fwd(v.flatten(1), w=w, b=b, Y=dO.flatten(1))
        val = h.view(v.shape)
        kw = dict(scale=0.125, cu=cu, S_in=S)
        S_out = torch.empty_like(S)
        out, saved = binding.chela_gated_delta_fwd(q, k, val, g, beta, S_out=S_out, want_saved=True, **kw)
        d = binding.chela_gated_delta_bwd(q, k, val, g, beta, dO, dS_out=S_out, want_dS_in=True, saved=saved, **kw)
        e = binding.chela_gated_delta_bwd(q, k, val, g, beta, dO, **kw)
        n = binding.chela_layer_norm_bwd(X, d[2].flatten(1), w=w, want_db=True, dX_out=out.flatten(1))
        o = binding.chela_gated_delta_step(*(t[:3].contiguous() for t in (q, k, val, g, beta)), S_out)
        return [t for t in (X, h, out, S_out, o, *d, *e, *n) if t is not None]

    return run, (v, dO, beta)


def _runs():
    return [_training_pass(300, 4, 2, 64, 64, BF, 67), _training_pass(200, 2, 2, 128, 64, F32, 71)]


def _new_values(inputs, other):
    for t in inputs:
        y = other(*t.shape)
        t.copy_((torch.sigmoid(y) if t.dim() == 2 else y).to(t.dtype))


def test_on_other_streams_and_two_at_once():
    runs = [run for run, _ in _runs()]
    want = [run() for run in runs]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in runs], [[], []]
    for _ in range(2):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(runs[i]())
    torch.cuda.synchronize()
    for w, g in zip(want, got):
        for one in g:
            for p, q in zip(w, one):
                assert torch.equal(p, q)
    # a stream that is named
    s = torch.cuda.Stream()
    x = inputs(gen(3), 100, 2, 2, 64, 64, BF)
    a = binding.chela_gated_delta_fwd(*x[:5])[0]
    s.wait_stream(torch.cuda.current_stream())
    b = binding.chela_gated_delta_fwd(*x[:5], stream=s)[0]
    s.synchronize()
    assert torch.equal(a, b)


@pytest.mark.parametrize("own_scratch", [False, True])
def test_captured_and_replayed(own_scratch):
    # two graphs; with the library's own scratch they share their stream's
    runs = _runs()
    ws = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")
    s, graphs, outs = torch.cuda.Stream(), [], []
    if not own_scratch:
        binding.chela_set_workspace(ws)
    try:
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            for run, _ in runs:
                run()
        torch.cuda.current_stream().wait_stream(s)
        for run, _ in runs:
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=s):
                outs.append(run())
            graphs.append(g)
    finally:
        binding.chela_set_workspace(None)
    other = gen(73)
    for k in range(4):
        for _, inp in runs:
            _new_values(inp, other)
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


def test_runs_captured_and_replayed_with_other_offsets():
    T, H = 1600, 2
    x = inputs(gen(37), T, H, H, 64, 64, BF)
    cu = cu_of([1500, 100])

    def run():
        out, saved = binding.chela_gated_delta_fwd(*x[:5], cu=cu, want_saved=True)
        return [out, *binding.chela_gated_delta_bwd(*x, cu=cu, saved=saved)[:5], *binding.chela_gated_delta_bwd(*x, cu=cu)[:5],
                binding.chela_gated_delta_fwd(*x[:5], cu=cu)[0]]

    s, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        run()
    torch.cuda.current_stream().wait_stream(s)
    with torch.cuda.graph(g, stream=s):
        got = run()
    for lens in ([800, 800], [1600, 0], [3, 1590], [1500, 100], [0, 1]):
        cu.copy_(cu_of(lens))
        want = run()
        for t in got:
            t.fill_(float("nan"))
        g.replay()
        torch.cuda.synchronize()
        for p, q in zip(got, want):
            assert torch.equal(p, q), lens
        check_all(dict(O=got[0], dV=got[3], dK=got[2]), x, None, None, lens, 1.0, BF, bounds=False)


def test_two_threads_with_streams_of_their_own():
    import threading
    runs = [run for run, _ in _runs()]
    want = [run() for run in runs]
    torch.cuda.synchronize()
    got, wrong = [None, None], []

    def work(i):
        try:
            s = torch.cuda.Stream()
            with torch.cuda.stream(s):
                for _ in range(5):
                    got[i] = runs[i]()
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


@pytest.mark.parametrize("dtype", DTYPES)
def test_the_compiled_host_path_and_the_binding_do_the_same(dtype):
    # (with a stream named, a call goes through the binding's own lines)
    r, H, Hk, dk, dv, n, L = gen(61), 4, 2, 64, 128, 3, 40
    here = torch.cuda.current_stream()
    x = inputs(r, n * L, H, Hk, dk, dv, dtype)
    b4 = [t.view(n, L, *t.shape[1:]) for t in x]
    wide = [wide_rows(t, 1) for t in x]
    cu, slots = cu_of([20, 0, 70, 25]), torch.tensor([1, 3, 2, 0], dtype=torch.int32, device="cuda")
    pool = r(5, H, dk, dv)

    def both(f, *args, states=(), **kw):
        out = []
        for s in (None, here):
            own = {k: v.clone() for k, v in states}
            kw = {k: v.clone() if k in ("O", "o") else v for k, v in kw.items()}
            if "S_in" in own:
                own["S_out"] = own["S_in"]
            y = f(*args, stream=s, **own, **kw)
            out.append([t for t in (y if isinstance(y, tuple) else (y,)) if t is not None] + list(own.values()))
        assert len(out[0]) == len(out[1])
        for a, b in zip(*out):
            if a.dtype == F32 and a.dim() == 1 and f is binding.chela_gated_delta_fwd:
                assert a.shape == b.shape                          # (what is saved: places that no chunk has hold anything)
                continue
            assert a.shape == b.shape and a.dtype == b.dtype and torch.equal(a, b)

    fwd, bwd, step = binding.chela_gated_delta_fwd, binding.chela_gated_delta_bwd, binding.chela_gated_delta_step
    nog = lambda t: [*t[:3], None, t[4]]  # noqa: E731
    for t in (x, b4, wide):
        both(fwd, *t[:5], scale=0.5)
        both(bwd, *t[:5], t[5], scale=0.5)
        both(fwd, *nog(t))
        both(bwd, *nog(t), t[5])
    both(fwd, *x[:5], cu=cu, states=[("S_in", pool)], slots=slots, want_saved=True, O=torch.zeros_like(x[2]))
    saved = fwd(*x[:5], cu=cu, S_in=pool[:4], want_saved=True)[1]
    both(bwd, *x[:5], x[5], cu=cu, S_in=pool[:4], dS_out=pool[:4], want_dS_in=True, saved=saved)
    five = torch.tensor([0, -1, 2, 4, 1], dtype=torch.int32, device="cuda")
    both(step, *(t[:5] for t in x[:5]), states=[("S", pool)], slots=five, o=torch.zeros_like(x[2][:5]))
    both(step, *(t[:5] for t in wide[:5]), states=[("S", pool)], scale=2.0)
    for bad in (dict(saved=saved[:-4]), dict(saved=saved.double()), dict(dS_out=pool), dict(S_in=pool.double()), dict(cu=cu.long())):
        for s in (None, here):
            with pytest.raises(ValueError):
                bwd(*x[:5], x[5], **dict(dict(cu=cu, stream=s), **bad))
    for s in (None, here):
        with pytest.raises(ValueError):
            fwd(x[0], x[1][:, :1], *x[2:5], stream=s)
        with pytest.raises(ValueError):
            fwd(x[0], x[1], x[2], x[3][:, :1], x[4], stream=s)
        with pytest.raises(ValueError):
            fwd(x[0].double(), *x[1:5], stream=s)
        with pytest.raises(binding.ChelaError):
            fwd(x[0][..., :32].contiguous(), x[1][..., :32].contiguous(), *x[2:5], stream=s)
        with pytest.raises(binding.ChelaError):
            fwd(*x[:5], scale=float("nan"), stream=s)
    D = 96
    X, Y, w, dN = r(30, D).to(dtype), r(30, D).to(dtype), r(D), r(30, D).to(dtype)
    for kw in (dict(w=w, b=w, Y=Y), dict(Y=Y), dict(w=w), {}):
        both(binding.chela_layer_norm_fwd, X, **kw)
        both(binding.chela_layer_norm_fwd, X.float(), **kw)
    for kw in (dict(w=w, want_db=True, dX_out=Y), dict(want_db=True), dict(w=w), {}):
        both(binding.chela_layer_norm_bwd, X, dN, **kw)
    for s in (None, here):
        y = Y.clone()
        assert binding.chela_layer_norm_bwd(X, dN, dX_out=y, in_place=True, stream=s)[0] is y
        assert binding.chela_layer_norm_fwd(X, stream=s)[0] is X
        for bad in (dict(w=w[1:]), dict(Y=Y[1:]), dict(b=w.double())):
            with pytest.raises(ValueError):
                binding.chela_layer_norm_fwd(X, **dict(dict(stream=s), **bad))
        with pytest.raises(ValueError):
            binding.chela_layer_norm_bwd(X, dN, in_place=True, stream=s)


def test_gradients_against_differences():
    # fp32, along one random direction of all inputs: central differences of a loss in 64 bits of the outputs
    r, H, Hk, dk, dv, T = gen(91), 2, 1, 64, 64, 70
    x = list(inputs(r, T, H, Hk, dk, dv, F32))
    dO, S, dS = x.pop(), 0.3 * r(1, H, dk, dv), 0.3 * r(1, H, dk, dv)
    leaves = x + [S]
    way = [r(*t.shape) for t in leaves]
    way = [d / max(d.norm(), 1e-9) * t.norm() for d, t in zip(way, leaves)]
    g = binding.chela_gated_delta_bwd(*x, dO, S_in=S, dS_out=dS, want_dS_in=True)
    slope = sum((a.double() * d.double()).sum() for a, d in zip(g, way))

    def loss(h):
        y = [t + h * d for t, d in zip(leaves, way)]
        S_out = torch.empty_like(S)
        out = binding.chela_gated_delta_fwd(*y[:5], S_in=y[5], S_out=S_out)[0]
        return (out.double() * dO.double()).sum() + (S_out.double() * dS.double()).sum()

    # the difference's truncation goes with h^2, the fp32 outputs' roundings (2e-6 of their size, as above) with 1 / h: Richardson's two sizes
    d1, d2 = ((loss(h) - loss(-h)) / (2 * h) for h in (2e-3, 4e-3))
    better = (4 * d1 - d2) / 3
    size = (dO.double().norm() + dS.double().norm()) * 30
    assert abs(better - slope) <= 1e-3 * abs(slope) + 4e-6 * size / 2e-3, (better, slope)


def test_offsets_beyond_32_bits():
    # rows, and a pool of states, behind 2^31 elements
    r, H, dk, dv = gen(47), 1, 64, 64
    T, wide = 40, 1 << 26
    big = torch.zeros(T, wide, dtype=BF, device="cuda")                    # 2.7e9 elements
    v = big[:, -H * dv:].unflatten(1, (H, dv))
    q, k, vals, g, beta, dO = inputs(r, T, H, 1, dk, dv, BF)
    v.copy_(vals)
    a = binding.chela_gated_delta_fwd(q, k, v, g, beta)[0]
    b = binding.chela_gated_delta_fwd(q, k, vals, g, beta)[0]
    assert torch.equal(a, b)
    x = binding.chela_gated_delta_bwd(q, k, v, g, beta, v)
    y = binding.chela_gated_delta_bwd(q, k, vals, g, beta, vals)
    assert all(torch.equal(p, w) for p, w in zip(x[:5], y[:5]))
    del big, v
    n = (1 << 31) // (dk * dv) + 4
    pool = torch.zeros(n, H, dk, dv, device="cuda")
    st = 0.3 * r(2, H, dk, dv)
    pool[-2:] = st
    slots = torch.tensor([n - 2, n - 1], dtype=torch.int32, device="cuda")
    cu = cu_of([13, 27])
    a = binding.chela_gated_delta_fwd(q, k, vals, g, beta, cu=cu, S_in=pool, S_out=pool, slots=slots)[0]
    S_out = torch.empty_like(st)
    b = binding.chela_gated_delta_fwd(q, k, vals, g, beta, cu=cu, S_in=st, S_out=S_out)[0]
    assert torch.equal(a, b) and torch.equal(pool[-2:], S_out)
    a = binding.chela_gated_delta_step(*(t[:2] for t in (q, k, vals, g, beta)), pool, slots=slots)
    b = binding.chela_gated_delta_step(*(t[:2] for t in (q, k, vals, g, beta)), S_out)
    assert torch.equal(a, b) and torch.equal(pool[-2:], S_out) and (pool[:4] == 0).all()
