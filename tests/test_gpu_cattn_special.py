"""Causal attention with values that are not finite, in calls of every cut: they reach those who see them, as the formulas
say, and nobody else; and the same calls without them against the fp64 oracle where that is affordable.

Bound between two runs: each is within the bounds of test_gpu_cattn.py of the exact result, so they are within twice those of each
other (a wavefront that meets such values forms its sums another way)."""
import numpy as np
import pytest

from oracle import vfm_oracle as orc
from paper_2503_12964_amd import workloads as W
from tests import parity_utils as U

pytestmark = pytest.mark.gpu


def _binding():
    from paper_2503_12964_amd import binding
    binding.load_library()
    return binding


def _cu(lens):
    return np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)


def _inputs(q, kv, heads, kvh, hd, seed):
    tq, tk = sum(q), sum(kv)
    draw = lambda name, shape: U.to_device(W.f32_to_bf16_bits(W.normal_f32(seed, name, shape, 1.0)))  # noqa: E731
    return {"q": draw("q", (tq, heads, hd)), "k": draw("k", (tk, kvh, hd)), "v": draw("v", (tk, kvh, hd)), "dout": draw("dout", (tq, heads, hd))}


def _run(dev, cq, ck, scale):
    b = _binding()
    out, lse = b.vfm_cattn_fwd(dev["q"], dev["k"], dev["v"], cq, ck, scale)
    dq, dk, dv = b.vfm_cattn_bwd(dev["q"], dev["k"], dev["v"], out, lse, dev["dout"], cq, ck, scale)
    return {"out": out, "lse": lse, "dq": dq, "dk": dk, "dv": dv}


# queries, keys, heads, kv heads: few rows and many, whole tiles and cut ones, one K/V head and several
CALLS = {
    "small": ((37, 5, 80), (37, 5, 80), 4, 2),
    "queries_without_keys": ((40, 33, 70), (17, 1, 69), 6, 2),
    "sixteen_to_one": ((130, 45), (130, 45), 16, 1),
    "one_sequence": ((1500,), (1500,), 4, 2),
    "one_long_to_one": ((2600,), (2600,), 8, 1),
    "many": ((260,) * 24, (260,) * 24, 16, 4),
    "many_heads": ((700, 333) * 3, (700, 333) * 3, 32, 8),
    "chunk": ((64, 1), (2900, 700), 8, 2),
    "wide_chunk": ((300, 170), (2000, 170), 12, 4),
}


def _places(q, kv, rng):
    """A query of every sequence and a key that it sees and the ones before it do not, somewhere within."""
    picks = []
    for s, (n, m) in enumerate(zip(q, kv)):
        lo = max(0, n - m)
        if n > lo:
            i = int(rng.integers(lo, n))
            picks.append((s, i, i + m - n))
    return picks


def _compare(name, got, clean, bad, tol):
    """bad: what may not be finite, and has to be so; the rest is as without."""
    g, c = U.to_f64(got), U.to_f64(clean)
    assert np.array_equal(np.isfinite(g) | np.isneginf(c), ~bad), name
    g, c = np.where(bad | np.isneginf(c), 0.0, g), np.where(bad | np.isneginf(c), 0.0, c)
    if name == "lse":
        assert U.max_abs(g, c) <= 2 * tol
    elif c.any():
        U.assert_rows_close(name, g, c, 2 * tol, tensor_rms=10 * float(np.sqrt(np.mean(c * c))))


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("where", ["k", "v", "q", "dout"])
@pytest.mark.parametrize("name", list(CALLS))
def test_what_is_not_finite_reaches_those_who_see_it(name, where, hd):
    q, kv, heads, kvh = CALLS[name]
    cq, ck, scale, group = _cu(q), _cu(kv), hd ** -0.5, heads // kvh
    dev = _inputs(q, kv, heads, kvh, hd, 80 + hd)
    clean = _run(dev, cq, ck, scale)
    rng = np.random.default_rng(len(name))
    bad = {n: np.zeros(tuple(t.shape), dtype=bool) for n, t in clean.items()}
    for x, (s, i, j) in enumerate(_places(q, kv, rng)):
        n, d = int(rng.integers(kvh)), int(rng.integers(hd))
        h = n * group + int(rng.integers(group))
        value = float("nan") if where in ("k", "q") or x % 2 else float("inf")
        rows, seen, mine = slice(cq[s] + i, cq[s + 1]), slice(ck[s], ck[s] + j + 1), slice(n * group, (n + 1) * group)
        keys = slice(ck[s], ck[s + 1])
        if where in ("k", "v"):
            dev[where][ck[s] + j, n, d] = value
            bad["out"][rows, mine, d if where == "v" else slice(None)] = True
            bad["dq"][rows, mine] = True
            bad["dk"][keys, n] = True                       # (the last query sees all keys, the bad one among them)
            if where == "k":
                bad["lse"][mine, rows] = True
                bad["dv"][keys, n] = True
        else:
            dev[where][cq[s] + i, h, d] = value
            bad["dq"][cq[s] + i, h] = True
            bad["dk"][seen, n] = True
            if where == "q":
                bad["out"][cq[s] + i, h] = True
                bad["lse"][h, cq[s] + i] = True
                bad["dv"][seen, n] = True
            else:
                bad["dv"][seen, n, d] = True
    for s, (n, m) in enumerate(zip(q, kv)):                 # queries that see nothing: whatever they hold
        if n > m:
            dev["q" if where != "dout" else where][cq[s]:cq[s] + n - m] = float("nan")
    got = _run(dev, cq, ck, scale)
    for n, tol in (("out", U.TOL_OUT_RELRMS), ("lse", U.TOL_LSE_MAXABS), ("dq", U.TOL_GRAD_RELRMS), ("dk", U.TOL_GRAD_RELRMS),
                   ("dv", U.TOL_GRAD_RELRMS)):
        _compare(n, got[n], clean[n], bad[n], tol)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("where", ["q", "k", "v", "dout"])
def test_all_of_it_not_finite(where, hd):
    """A tensor that has become NaN altogether: whoever sees a key gets NaN, and the call ends soon."""
    q, kv, heads, kvh = (300, 40), (300, 20), 8, 2
    cq, ck, scale = _cu(q), _cu(kv), hd ** -0.5
    dev = _inputs(q, kv, heads, kvh, hd, 90 + hd)
    clean = {n: U.to_f64(t) for n, t in _run(dev, cq, ck, scale).items()}
    dev[where].fill_(float("nan"))
    got = {n: U.to_f64(t) for n, t in _run(dev, cq, ck, scale).items()}
    some = np.isfinite(clean["lse"]).T
    touched = {"q": ("out", "dq", "dk", "dv"), "k": ("out", "dq", "dk", "dv"), "v": ("out", "dq", "dk"), "dout": ("dq", "dk", "dv")}[where]
    for n in ("out", "dq"):
        want = some if n in touched else np.zeros_like(some)
        assert np.array_equal(np.isnan(got[n]).all(axis=-1), want) and np.array_equal(np.isnan(got[n]).any(axis=-1), want), n
        assert not got[n][~some].any()
    for n in ("dk", "dv"):
        assert np.isnan(got[n]).all() if n in touched else np.isfinite(got[n]).all(), n


def _expected(host, cq, ck, scale, heads):
    """The oracle's results of one K/V head's query heads."""
    out, lse = orc.cattn_fwd(host["q"], host["k"], host["v"], cq, ck, scale)
    dq, dk, dv = orc.cattn_bwd(host["q"], host["k"], host["v"], host["dout"], cq, ck, scale)
    return {"out": out, "lse": lse, "dq": dq, "dk": dk, "dv": dv}


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("name", ["one_sequence", "one_long_to_one", "many", "many_heads", "chunk", "wide_chunk"])
def test_calls_of_every_cut(name, hd):
    q, kv, heads, kvh = CALLS[name]
    cq, ck, scale = _cu(q), _cu(kv), hd ** -0.5
    dev = _inputs(q, kv, heads, kvh, hd, 100 + hd)
    got = {n: U.to_f64(t) for n, t in _run(dev, cq, ck, scale).items()}
    group, n = heads // kvh, kvh - 1                        # (one K/V head: the oracle takes seconds a head)
    host = {x: U.to_f64(t) for x, t in dev.items()}
    mine = slice(n * group, (n + 1) * group)
    part = {"q": host["q"][:, mine], "dout": host["dout"][:, mine], "k": host["k"][:, n:n + 1], "v": host["v"][:, n:n + 1]}
    ref = _expected(part, cq, ck, scale, group)
    assert U.max_abs(got["lse"][mine], ref["lse"]) <= U.TOL_LSE_MAXABS
    for x, tol in (("out", U.TOL_OUT_RELRMS), ("dq", U.TOL_GRAD_RELRMS), ("dk", U.TOL_GRAD_RELRMS), ("dv", U.TOL_GRAD_RELRMS)):
        g = got[x][:, mine] if x in ("out", "dq") else got[x][:, n:n + 1]
        assert U.rel_rms(g, ref[x]) <= tol, (x, U.rel_rms(g, ref[x]))
        U.assert_rows_close(x, g, ref[x], tol, tensor_rms=10 * float(np.sqrt(np.mean(ref[x] * ref[x]))))
