"""Causal attention: an infinity stays an infinity where the formulas have one, and what overflows in a pair that is not seen (from
inputs that are all finite) has no part in any result.

Bound between two runs that differ only in what a row does not see: as in test_gpu_cattn_special.py, twice the bounds of
test_gpu_cattn.py, per row of the row's own magnitude or of a hundredth of its head's."""
import numpy as np
import pytest

from tests import parity_utils as U
from tests.test_gpu_cattn_special import CALLS, _binding, _cu, _inputs, _run

pytestmark = pytest.mark.gpu

BIG = 2.0 ** 80        # a product of two overflows fp32, one of them with values about 1 does not


def _same_rows(name, got, clean, rows):
    """got[rows] finite and as clean[rows]; rows: truth values over all axes but the last."""
    g, c = got[rows], clean[rows]
    assert np.isfinite(c).all(), name
    assert np.isfinite(g).all(), (name, int((~np.isfinite(g)).any(axis=-1).sum()), len(g))
    if c.any():
        U.assert_rows_close(name, g, c, 2 * U.TOL_GRAD_RELRMS, tensor_rms=10 * float(np.sqrt(np.median(np.mean(c * c, axis=-1)))))


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("at", ["middle", "last"])
@pytest.mark.parametrize("name", list(CALLS))
def test_an_infinite_element_of_dout_gives_infinities_in_dv(name, at, hd):
    """dv_jd = sum_i P_ij dO_id: one infinite term, its sign; every other column as without."""
    q, kv, heads, kvh = CALLS[name]
    cq, ck, scale, group = _cu(q), _cu(kv), hd ** -0.5, heads // kvh
    dev = _inputs(q, kv, heads, kvh, hd, 140 + hd)
    clean = U.to_f64(_run(dev, cq, ck, scale)["dv"])
    want = clean.copy()
    rng = np.random.default_rng(hd + len(name))
    for s, (n, m) in enumerate(zip(q, kv)):
        lo = max(0, n - m)
        if n == lo:
            continue
        i = (lo + n) // 2 if at == "middle" else n - 1
        x, d, sign = (kvh - 1 if at == "last" else int(rng.integers(kvh))), int(rng.integers(hd)), (1.0, -1.0)[s % 2]
        h = x * group + (group - 1 if at == "last" else int(rng.integers(group)))        # (the last row of all: copies stand past it)
        dev["dout"][cq[s] + i, h, d] = sign * float("inf")
        want[ck[s]:ck[s] + i + m - n + 1, x, d] = sign * np.inf
    got = U.to_f64(_run(dev, cq, ck, scale)["dv"])
    assert np.array_equal(np.isinf(want), np.isinf(got)) and np.array_equal(want[np.isinf(want)], got[np.isinf(want)])
    fin = np.isfinite(want)
    assert np.isfinite(got[fin]).all()
    U.assert_rows_close("dv", np.where(fin, got, 0.0), np.where(fin, clean, 0.0), 2 * U.TOL_GRAD_RELRMS,
                        tensor_rms=10 * float(np.sqrt(np.mean(clean * clean))))


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("at", ["middle", "last"])
@pytest.mark.parametrize("name", list(CALLS))
def test_an_infinite_element_of_v_gives_infinities_in_out(name, at, hd):
    q, kv, heads, kvh = CALLS[name]
    cq, ck, scale, group = _cu(q), _cu(kv), hd ** -0.5, heads // kvh
    dev = _inputs(q, kv, heads, kvh, hd, 150 + hd)
    clean = U.to_f64(_run(dev, cq, ck, scale)["out"])
    want = clean.copy()
    rng = np.random.default_rng(hd + len(name))
    for s, (n, m) in enumerate(zip(q, kv)):
        if n == 0 or m == 0:
            continue
        j = m // 2 if at == "middle" else m - 1
        x, d, sign = int(rng.integers(kvh)), int(rng.integers(hd)), (1.0, -1.0)[s % 2]
        dev["v"][ck[s] + j, x, d] = sign * float("inf")
        want[cq[s] + max(0, j - (m - n)):cq[s + 1], x * group:(x + 1) * group, d] = sign * np.inf
    got = U.to_f64(_run(dev, cq, ck, scale)["out"])
    assert np.array_equal(np.isinf(want), np.isinf(got)) and np.array_equal(want[np.isinf(want)], got[np.isinf(want)])
    fin = np.isfinite(want)
    assert np.isfinite(got[fin]).all()
    U.assert_rows_close("out", np.where(fin, got, 0.0), np.where(fin, clean, 0.0), 2 * U.TOL_OUT_RELRMS,
                        tensor_rms=10 * float(np.sqrt(np.mean(clean * clean))))


def _pairs(q, kv, rng):
    """Of every sequence a query with another before and after it, and the last key that it sees."""
    picks = []
    for s, (n, m) in enumerate(zip(q, kv)):
        lo = max(0, n - m) + 1
        if n - 1 > lo:
            i = int(rng.integers(lo, n - 1))
            picks.append((s, i, i + m - n))
    return picks


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("name", list(CALLS))
def test_a_delta_that_overflows_stays_with_the_keys_that_its_row_sees(name, hd):
    """Finite values throughout: a key's large value and a query's large dout that meet in Delta.  Keys after the query's last do not
    see it, and their dk, dv are those without the large dout; so is dq of every other query."""
    q, kv, heads, kvh = CALLS[name]
    cq, ck, scale, group = _cu(q), _cu(kv), hd ** -0.5, heads // kvh
    dev = _inputs(q, kv, heads, kvh, hd, 160 + hd)
    rng = np.random.default_rng(hd + len(name))
    picks = [(*p, int(rng.integers(heads))) for p in _pairs(q, kv, rng)]
    for s, i, j, h in picks:
        dev["v"][ck[s] + j, h // group] *= BIG
    clean = {n: U.to_f64(t) for n, t in _run(dev, cq, ck, scale).items()}
    others, after = np.ones((sum(q), heads), dtype=bool), np.ones((sum(kv), kvh), dtype=bool)
    for s, i, j, h in picks:
        dev["dout"][cq[s] + i, h] *= BIG
        others[cq[s] + i, h] = False
        after[ck[s]:ck[s] + j + 1, h // group] = False
    got = {n: U.to_f64(t) for n, t in _run(dev, cq, ck, scale).items()}
    for s, i, j, h in picks:
        assert not np.isfinite(got["dq"][cq[s] + i, h]).all()          # (the case is what it says)
    _same_rows("dq", got["dq"], clean["dq"], others)
    _same_rows("dk", got["dk"], clean["dk"], after)
    _same_rows("dv", got["dv"], clean["dv"], after)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("name", list(CALLS))
def test_products_of_unseen_pairs_may_overflow(name, hd):
    """A query's dout times the value of the key next after its last one is beyond fp32: neither meets the other's result."""
    q, kv, heads, kvh = CALLS[name]
    cq, ck, scale, group = _cu(q), _cu(kv), hd ** -0.5, heads // kvh
    base = _inputs(q, kv, heads, kvh, hd, 170 + hd)
    rng = np.random.default_rng(hd + len(name))
    picks = [(*p, int(rng.integers(heads))) for p in _pairs(q, kv, rng)]
    rows = np.ones((sum(q), heads), dtype=bool)            # that see no large value
    keys = np.ones((sum(kv), kvh), dtype=bool)             # that see no large dout

    def run(large_v, large_dout):
        dev = {n: t.clone() for n, t in base.items()}
        for s, i, j, h in picks:
            if large_v:
                dev["v"][ck[s] + j, h // group] *= BIG
                rows[cq[s] + i:cq[s + 1], h // group * group:(h // group + 1) * group] = False
            if large_dout:
                dev["dout"][cq[s] + i - 1, h] *= BIG
                keys[ck[s]:ck[s] + j, h // group] = False
        return {n: U.to_f64(t) for n, t in _run(dev, cq, ck, scale).items()}

    got, small_v, small_dout = run(True, True), run(False, True), run(True, False)
    _same_rows("out", got["out"], small_v["out"], rows)
    _same_rows("dq", got["dq"], small_v["dq"], rows)
    _same_rows("dk", got["dk"], small_dout["dk"], keys)
    _same_rows("dv", got["dv"], small_dout["dv"], keys)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("what", ["a query of NaN", "a column of infinities"])
def test_the_backward_stays_within_a_few_times_its_time(what, hd):
    """Sums that are formed again take their blocks straight from memory, without the loops' pipeline: some ten times the time of a
    block, for the wavefronts that met such values or for all of them.  25 leaves room for the clock; one pair at a time it
    was 50 to 80 times here, and more the longer the sequence."""
    import time
    import torch
    b = _binding()
    n, heads, kvh = 10000, 16, 4
    cu, scale = _cu((n,)), hd ** -0.5
    dev = _inputs((n,), (n,), heads, kvh, hd, 180 + hd)

    def best():
        out, lse = b.vfm_cattn_fwd(dev["q"], dev["k"], dev["v"], cu, cu, scale)
        times = []
        for _ in range(4):
            torch.cuda.synchronize()
            t = time.perf_counter()
            b.vfm_cattn_bwd(dev["q"], dev["k"], dev["v"], out, lse, dev["dout"], cu, cu, scale)
            torch.cuda.synchronize()
            times.append(time.perf_counter() - t)
        return min(times)

    clean = best()
    if what == "a query of NaN":
        dev["q"][n // 2, 3] = float("nan")
    else:
        dev["dout"][..., 5] = float("inf")
    taken = best()
    print(f"{what}, head_dim {hd}: {clean * 1e3:.2f} ms, {taken * 1e3:.2f} with it")
    assert taken <= 25 * clean
