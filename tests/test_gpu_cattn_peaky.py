"""Causal attention with scores of some tens in calls that are cut (pieces of one row's keys whose references differ by tens are joined,
shares of dK and dV added), and one sequence in packs of different company.

The gradients are compared with the formulas in 64 bits for the forward's own `out` and lse, as the backward is given them: Delta =
dout . out, or sum_j P dP for queries that see at most 32 keys.  (Against gradients from an exact out, its rounding in Delta alone would
be a per cent and more here: P is near 1, and dP - Delta small.)  What is left is the rounding of P or dS and of the result, half a
step of 2^-8 each, uniform in between: 2 * 2^-8 / sqrt(3) < 5e-3 in the RMS of a tensor."""
import numpy as np
import pytest

from oracle import vfm_oracle as orc
from tests import parity_utils as U
from tests.test_gpu_cattn_special import CALLS, _binding, _cu, _inputs

pytestmark = pytest.mark.gpu

TOL = 5e-3
# whether the forward is cut (a workspace tells), whether dK's and dV's sums are
CUT = {"one_sequence": (True, None), "one_long_to_one": (True, True), "chunk": (True, None), "wide_chunk": (True, None), "long_past": (True, None),
       "a_token_or_two": (True, None), "many_heads": (False, True), "many": (False, False), "two_long": (False, False)}


def _gradients(q, k, v, out, lse, dout, cq, ck, scale):
    """One K/V head: dq, dk, dv in 64 bits from the forward's out and lse."""
    dq, dk, dv = np.zeros_like(q), np.zeros_like(k), np.zeros_like(v)
    for s in range(len(cq) - 1):
        qs, ks = slice(cq[s], cq[s + 1]), slice(ck[s], ck[s + 1])
        n, m = cq[s + 1] - cq[s], ck[s + 1] - ck[s]
        if n == 0 or m == 0:
            continue
        seen = np.arange(m)[None] <= np.arange(n)[:, None] + m - n
        for h in range(q.shape[1]):
            S = scale * (q[qs, h] @ k[ks, 0].T)
            P = np.where(seen, np.exp(np.where(seen, S, 0.0) - np.where(np.isfinite(lse[h, qs]), lse[h, qs], 0.0)[:, None]), 0.0)
            dP = dout[qs, h] @ v[ks, 0].T
            delta = np.where(seen.sum(axis=1) <= 32, (P * dP).sum(axis=1), (dout[qs, h] * out[qs, h]).sum(axis=1))
            dS = P * (dP - delta[:, None])
            dq[qs, h] = scale * (dS @ k[ks, 0])
            dk[ks, 0] += scale * (dS.T @ q[qs, h])
            dv[ks, 0] += P.T @ dout[qs, h]
    return {"dq": dq, "dk": dk, "dv": dv}


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("name", list(CUT))
def test_scores_of_tens_in_calls_of_every_cut(name, hd):
    b = _binding()
    q, kv, heads, kvh = CALLS[name]
    cq, ck, scale = _cu(q), _cu(kv), hd ** -0.5
    fwd_cut, bwd_cut = CUT[name]
    assert (b.vfm_cattn_fwd_workspace_size(cq, ck, heads, kvh, hd) > 0) is fwd_cut
    if bwd_cut is not None:
        assert (b.vfm_cattn_bwd_workspace_size(cq, ck, heads, kvh, hd) > 8 * sum(q) * heads + 4096) is bwd_cut   # (more than Delta and lse)
    dev = _inputs(q, kv, heads, kvh, hd, 200 + hd)
    for n in ("q", "k"):
        dev[n] *= 3
    out, lse = b.vfm_cattn_fwd(dev["q"], dev["k"], dev["v"], cq, ck, scale)
    grads = b.vfm_cattn_bwd(dev["q"], dev["k"], dev["v"], out, lse, dev["dout"], cq, ck, scale)
    group, n = heads // kvh, kvh - 1                           # (one K/V head: the oracle takes seconds a head)
    mine = slice(n * group, (n + 1) * group)
    host = {x: U.to_f64(t)[:, mine if x in ("q", "dout") else slice(n, n + 1)] for x, t in dev.items()}
    o, l = U.to_f64(out)[:, mine], U.to_f64(lse)[mine]
    o_ref, l_ref = orc.cattn_fwd(host["q"], host["k"], host["v"], cq, ck, scale)
    assert U.max_abs(l, l_ref) <= U.TOL_LSE_MAXABS
    assert U.rel_rms(o, o_ref) <= TOL
    U.assert_rows_close("out", o, o_ref, TOL)
    ref = _gradients(host["q"], host["k"], host["v"], o, l, host["dout"], cq, ck, scale)
    for x, g in zip(("dq", "dk", "dv"), grads):
        g = U.to_f64(g)[:, mine if x == "dq" else slice(n, n + 1)]
        assert U.rel_rms(g, ref[x]) <= TOL, (x, U.rel_rms(g, ref[x]))
        U.assert_rows_close(x, g, ref[x], TOL, tensor_rms=10 * float(np.sqrt(np.mean(ref[x] * ref[x]))))


@pytest.mark.parametrize("hd", [64, 128])
def test_a_sequence_in_packs_of_different_company(hd):
    """Alone (cut), beside a short one, among many: each run is within its bounds of the exact result, so any two are within twice those."""
    import torch
    b = _binding()
    n, heads, kvh, scale = 2100, 8, 2, hd ** -0.5
    own = _inputs((n,), (n,), heads, kvh, hd, 210 + hd)
    alone, cuts = None, set()
    for company in ((), (5,), (900, 2000), (300,) * 70):
        other = _inputs(company, company, heads, kvh, hd, 211) if company else None
        dev = {x: t if other is None else torch.cat((other[x], t)) for x, t in own.items()}
        cu = _cu((*company, n))
        cuts.add(b.vfm_cattn_fwd_workspace_size(cu, cu, heads, kvh, hd) > 0)
        out, lse = b.vfm_cattn_fwd(dev["q"], dev["k"], dev["v"], cu, cu, scale)
        got = (out, *b.vfm_cattn_bwd(dev["q"], dev["k"], dev["v"], out, lse, dev["dout"], cu, cu, scale))
        got = [U.to_f64(t[-n:]) for t in got]
        lse = U.to_f64(lse[:, -n:])
        if alone is None:
            alone = (got, lse)
            continue
        assert U.max_abs(lse, alone[1]) <= 2 * U.TOL_LSE_MAXABS
        for x, g, a, tol in zip(("out", "dq", "dk", "dv"), got, alone[0], (U.TOL_OUT_RELRMS, *[U.TOL_GRAD_RELRMS] * 3)):
            U.assert_rows_close(x, g, a, 2 * tol, tensor_rms=10 * float(np.sqrt(np.mean(a * a))))
    assert cuts == {True, False}
