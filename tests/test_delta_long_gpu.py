"""The gated delta rule over runs of several chunks on the GPU, against the definition in 64 bits: decays above zero.

Tolerances, before any run.  By norms, over a sequence and head, as for decays below zero (test_delta_gpu.by_norm), times what a chunk lets grow: the
operands of its products are rounded relative to their size, which is up to e^(sum of the chunk's positive log decays) times that of what comes out
where keys replace what has grown.  How long the sequence is, and how many chunks a run has, does not come into it."""
import numpy as np
import pytest
import torch

from oracle import delta as R
from paper_2406_08128_amd import binding
from test_delta_gpu import BF, DTYPES, HALF, f64, gen

pytestmark = pytest.mark.gpu


def grown(what, got, ref, dtype, state, growth):
    rel = 2.0 ** -24 * 4 * np.sqrt(12 * 128)
    if dtype == BF:
        rel += 2.0 ** -16 * np.sqrt(6) if state else 2.0 ** -8 * np.sqrt(8)
    assert torch.isfinite(got).all(), what
    off = np.linalg.norm(f64(got) - ref)
    assert off <= (rel * growth + HALF[got.dtype]) * np.linalg.norm(ref), (what, off / np.linalg.norm(ref), rel * growth)


# Keys at right angles in turn, each token replacing what is at its key, while everything grows: what a key has is at most `period` tokens old and the
# state stays of the size of e^(period g).  Lengths for runs of 2 to 16 chunks.
GROWTH = [(64, 64, 16448, 0.02), (64, 64, 16448, 0.05), (64, 128, 4224, 0.02), (128, 128, 16500, 0.02), (128, 128, 33000, 0.01), (128, 64, 1100, 0.03)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("dk,dv,L,g", GROWTH)
def test_growth_that_keys_replace(dtype, dk, dv, L, g):
    r = gen(dk + dv + L)
    k = torch.eye(dk, device="cuda")[torch.arange(L, device="cuda") % dk][:, None].to(dtype)
    q, v, dO = (r(L, 1, dk) / dk ** 0.5).to(dtype), r(L, 1, dv).to(dtype), r(L, 1, dv).to(dtype)
    g = torch.full((L, 1), g, device="cuda").to(dtype)
    beta = torch.ones(L, 1, device="cuda").to(dtype)
    growth = float(np.exp(f64(g)[0, 0] * (64 if dtype == BF else 32)))
    x = (q, k, v, g, beta)
    args = [f64(t)[:, 0] for t in x]
    ref = dict(zip(("O", "S_out"), R.delta_fwd(*args)))
    ref.update(R.delta_bwd(*args, f64(dO)[:, 0]))
    S_out = torch.empty(1, 1, dk, dv, device="cuda")
    for kept, out in ((False, None), (True, None), (False, S_out)):
        O, saved = binding.chela_gated_delta_fwd(*x, want_saved=kept, S_out=out)
        grown(("O", kept, out is None), O[:, 0], ref["O"], dtype, False, growth)
        if out is not None:
            grown("S_out", S_out[0, 0], ref["S_out"], dtype, True, growth)
        for s in ((saved, None) if kept else ()):
            grads = binding.chela_gated_delta_bwd(*x, dO, saved=s)
            for n, t in zip(("dQ", "dK", "dV", "dbeta"), (*grads[:3], grads[4])):
                grown((n, s is None), t[:, 0], ref[n], dtype, False, growth)


@pytest.mark.parametrize("dtype", DTYPES)
def test_decay_behind_growth_and_growth_behind_decay(dtype):
    # a few hundred tokens of either in turn, so that runs have both; keys in turn, three quarters of what is at a key replaced
    r, L, d = gen(7), 16448, 64
    q = torch.nn.functional.normalize(r(L, 1, d), dim=-1).to(dtype)
    k = torch.eye(d, device="cuda")[torch.arange(L, device="cuda") * 5 % d][:, None].to(dtype)
    v, dO = r(L, 1, d).to(dtype), r(L, 1, d).to(dtype)
    g = torch.where(torch.arange(L, device="cuda") // 200 % 2 == 0, 0.015625, -0.25)[:, None].to(dtype)
    beta = torch.full((L, 1), 0.75, device="cuda").to(dtype)
    x = (q, k, v, g, beta)
    args = [f64(t)[:, 0] for t in x]
    growth = float(np.exp(0.015625 * (64 if dtype == BF else 32)))
    ref = dict(zip(("O", "S_out"), R.delta_fwd(*args)))
    ref.update(R.delta_bwd(*args, f64(dO)[:, 0]))
    S_out = torch.empty(1, 1, d, d, device="cuda")
    grown("O", binding.chela_gated_delta_fwd(*x)[0][:, 0], ref["O"], dtype, False, growth)
    binding.chela_gated_delta_fwd(*x, S_out=S_out)
    grown("S_out", S_out[0, 0], ref["S_out"], dtype, True, growth)
    for n, t in zip(("dQ", "dK", "dV"), binding.chela_gated_delta_bwd(*x, dO)):
        grown(n, t[:, 0], ref[n], dtype, False, growth)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("dk,dv", [(64, 64), (128, 128)])
def test_growth_chunk_by_chunk_with_states(dtype, dk, dv):
    r, L, share = gen(dk), 1100, 2
    k = torch.eye(dk, device="cuda")[torch.arange(L, device="cuda") * 3 % dk][:, None].to(dtype)
    q, v, dO = (r(L, 1, dk) / dk ** 0.5).to(dtype), r(L, share, dv).to(dtype), r(L, share, dv).to(dtype)
    g = torch.full((L, share), 0.03125, device="cuda").to(dtype)
    beta = torch.ones(L, share, device="cuda").to(dtype)
    S, dS, S_out = 0.3 * r(1, share, dk, dv), 0.3 * r(1, share, dk, dv), torch.empty(1, share, dk, dv, device="cuda")
    growth = float(np.exp(0.03125 * (64 if dtype == BF else 32)))
    O, saved = binding.chela_gated_delta_fwd(q, k, v, g, beta, S_in=S, S_out=S_out, want_saved=True)
    for s in (saved, None):
        grads = binding.chela_gated_delta_bwd(q, k, v, g, beta, dO, S_in=S, dS_out=dS, want_dS_in=True, saved=s)
        sums = [0, 0]
        for h in range(share):
            args = [f64(t)[:, 0 if i < 2 else h] for i, t in enumerate((q, k, v, g, beta))]
            ref = dict(zip(("O", "S_out"), R.delta_fwd(*args, state=f64(S)[0, h])))
            ref.update(R.delta_bwd(*args, f64(dO)[:, h], state=f64(S)[0, h], dstate=f64(dS)[0, h]))
            grown("O", O[:, h], ref["O"], dtype, False, growth)
            grown("S_out", S_out[0, h], ref["S_out"], dtype, True, growth)
            grown("dV", grads[2][:, h], ref["dV"], dtype, False, growth)
            grown("dS_in", grads[5][0, h], ref["dS_in"], dtype, True, growth)
            sums = [a + ref[n] for a, n in zip(sums, ("dQ", "dK"))]
        for n, t, a in zip(("dQ", "dK"), grads, sums):
            grown(n, t[:, 0], a, dtype, False, growth)
