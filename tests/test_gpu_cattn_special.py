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
    "a_token_or_two": ((2, 1), (2900, 700), 8, 2),
    "drafts": ((12, 9), (2500, 100), 8, 2),
    "long_past": ((1000,), (8000,), 16, 2),
    "two_long": ((2048, 1900), (2048, 1900), 32, 8),
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
@pytest.mark.parametrize("name", [n for n in CALLS if n not in ("small", "queries_without_keys", "sixteen_to_one")])
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


@pytest.mark.parametrize("hd", [64, 128])
def test_graphs_that_share_a_workspace(hd):
    """Two captured training steps of different cuts on one workspace, replayed in turn with eager work between, on changing inputs;
    and the same calls on a stream of the caller's."""
    import torch
    b = _binding()
    scale = hd ** -0.5
    calls = []
    for x, name in enumerate(("one_long_to_one", "chunk", "wide_chunk")):
        q, kv, heads, kvh = CALLS[name]
        cq, ck = _cu(q), _cu(kv)
        dev = _inputs(q, kv, heads, kvh, hd, 110 + x)
        need = [f(cq, ck, heads, kvh, hd) for f in (b.vfm_cattn_fwd_workspace_size, b.vfm_cattn_bwd_workspace_size)]
        calls.append((dev, cq, ck, need, heads))
    assert any(c[3][0] for c in calls)                      # (the forward's cut needs one)
    ws = torch.empty(max(max(c[3]) for c in calls), dtype=torch.uint8, device="cuda")

    def step(c, got):
        dev, cq, ck = c[:3]
        b.vfm_cattn_fwd(dev["q"], dev["k"], dev["v"], cq, ck, scale, out=got["out"], lse=got["lse"], workspace=ws)
        b.vfm_cattn_bwd(dev["q"], dev["k"], dev["v"], got["out"], got["lse"], dev["dout"], cq, ck, scale, got["dq"], got["dk"], got["dv"],
                        workspace=ws)

    results, graphs = [], []
    for c in calls:
        dev = c[0]
        got = {"out": torch.zeros_like(dev["q"]), "lse": torch.zeros((c[4], dev["q"].shape[0]), device="cuda"), "dq": torch.zeros_like(dev["q"]),
               "dk": torch.zeros_like(dev["k"]), "dv": torch.zeros_like(dev["v"])}
        step(c, got)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step(c, got)
        results.append(got)
        graphs.append(graph)
    side = torch.cuda.Stream()
    for turn in range(3):
        ws.fill_(255)                                       # (as floats: NaN)
        wants = [_run(c[0], c[1], c[2], scale) for c in calls]
        for got in results:
            for t in got.values():
                t.zero_()
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for got, want in zip(results, wants):
            assert all(torch.equal(got[n], want[n]) for n in want)
        dev, cq, ck = calls[turn][:3]
        out, lse = b.vfm_cattn_fwd(dev["q"], dev["k"], dev["v"], cq, ck, scale, stream=side)
        grads = b.vfm_cattn_bwd(dev["q"], dev["k"], dev["v"], out, lse, dev["dout"], cq, ck, scale, stream=side)
        side.synchronize()
        assert all(torch.equal(x, wants[turn][n]) for x, n in zip((out, lse, *grads), ("out", "lse", "dq", "dk", "dv")))
        for c in calls:
            for t in c[0].values():
                t.mul_(0.75)
        torch.cuda.synchronize()


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("where", ["v", "dout"])
def test_one_column_not_finite(where, hd):
    """One element of every value, or of every row of dout: out's (dv's) other columns are as without."""
    q, kv, heads, kvh = CALLS["one_long_to_one"]
    cq, ck, scale = _cu(q), _cu(kv), hd ** -0.5
    dev = _inputs(q, kv, heads, kvh, hd, 120 + hd)
    clean = _run(dev, cq, ck, scale)
    dev[where][..., 37] = float("nan")
    got = _run(dev, cq, ck, scale)
    bad = {n: np.zeros(tuple(t.shape), dtype=bool) for n, t in clean.items()}
    bad["dq"][:] = bad["dk"][:] = True
    bad["out" if where == "v" else "dv"][..., 37] = True
    for n, tol in (("out", U.TOL_OUT_RELRMS), ("lse", U.TOL_LSE_MAXABS), ("dq", U.TOL_GRAD_RELRMS), ("dk", U.TOL_GRAD_RELRMS),
                   ("dv", U.TOL_GRAD_RELRMS)):
        _compare(n, got[n], clean[n], bad[n], tol)
