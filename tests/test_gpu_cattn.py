"""GPU parity of causal attention with grouped heads (forward and backward) against the fp64 oracle.

Bounds.  Forward: P is rounded to bf16 before the second product and out after it, half a step each, at most 2^-8
relative per term and uniform in between (RMS 2^-8 / sqrt(3) for values spread over a binade, 2^-8 at worst): the two
together stay under 5e-3 in the RMS of a tensor.  Backward: P or dS and the result are rounded likewise, and dS = P (dP - Delta)
carries the rounding of `out` in Delta: three roundings, 3 * 2^-8 / sqrt(3) < 1.5e-2.  lse is fp32 from exact products: 1e-3.
Per row: three times the tensor's bound of the row's own RMS, or of a hundredth of the tensor's for rows that are
small by cancellation (a query that sees one key has dq = 0: P is 1 within a few 2^-20, so dS is that share of dP, which is
up to 2^4, where the tensor's dq is dP times about 1 / sqrt(keys))."""
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


def _draw(seed, name, shape, gain=1.0):
    return W.f32_to_bf16_bits(W.normal_f32(seed, name, shape, gain))


def _inputs(q, kv, heads, kvh, hd, seed, gain=1.0):
    tq, tk = sum(q), sum(kv)
    bits = {"q": _draw(seed, "q", (tq, heads, hd), gain), "k": _draw(seed, "k", (tk, kvh, hd), gain),
            "v": _draw(seed, "v", (tk, kvh, hd)), "dout": _draw(seed, "dout", (tq, heads, hd))}
    return {n: U.to_device(x) for n, x in bits.items()}


def _assert_close(dev, out, lse, grads, cq, ck, scale):
    host = {n: U.to_f64(t) for n, t in dev.items()}
    o_ref, l_ref = orc.cattn_fwd(host["q"], host["k"], host["v"], cq, ck, scale)
    o, l = U.to_f64(out), U.to_f64(lse)
    assert np.array_equal(np.isneginf(l), np.isneginf(l_ref))
    some = np.isfinite(l_ref)
    assert U.max_abs(l[some], l_ref[some]) <= U.TOL_LSE_MAXABS
    assert not o[~some.T].any()
    assert U.rel_rms(o, o_ref) <= U.TOL_OUT_RELRMS
    U.assert_rows_close("out", o, o_ref, U.TOL_OUT_RELRMS)
    if grads is None:
        return
    for name, g, ref in zip(("dq", "dk", "dv"), grads, orc.cattn_bwd(host["q"], host["k"], host["v"], host["dout"], cq, ck, scale)):
        got = U.to_f64(g)
        assert np.all(np.isfinite(got)), name
        if not ref.any():      # nothing seen, or one key at most: exactly, or up to P's fp32 rounding, zero
            assert np.max(np.abs(got), initial=0.0) <= 2.0 ** -12, name
            continue
        U.assert_rows_close(name, got, ref, U.TOL_GRAD_RELRMS, tensor_rms=10 * float(np.sqrt(np.mean(ref * ref))))
        if np.max(np.diff(ck)) > 1 or name == "dv":
            assert U.rel_rms(got, ref) <= U.TOL_GRAD_RELRMS, (name, U.rel_rms(got, ref))


def _check(q, kv, heads, kvh, hd, seed=0, gain=1.0):
    b = _binding()
    cq, ck = _cu(q), _cu(kv)
    dev = _inputs(q, kv, heads, kvh, hd, seed, gain)
    scale = hd ** -0.5
    out, lse = b.vfm_cattn_fwd(dev["q"], dev["k"], dev["v"], cq, ck, scale)
    grads = b.vfm_cattn_bwd(dev["q"], dev["k"], dev["v"], out, lse, dev["dout"], cq, ck, scale)
    _assert_close(dev, out, lse, grads, cq, ck, scale)
    return dev, out, lse, grads


SELF = {
    "one_token": ((1,), 1, 1),
    "every_length_to_forty": (tuple(range(0, 41)), 3, 1),
    "around_units": ((31, 32, 33, 63, 64, 65, 127, 128, 129), 4, 2),
    "around_tiles": ((255, 256, 257, 1, 0, 300), 6, 2),
    "seven_to_one": ((200, 3, 77), 7, 1),
    "sixteen_to_one": ((130, 45), 16, 1),
    "one_to_one": ((513, 100), 3, 3),
    "over_a_thousand": ((1100, 90), 2, 1),
}


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("name", list(SELF))
def test_self_attention(name, hd):
    lens, heads, kvh = SELF[name]
    _check(lens, lens, heads, kvh, hd, seed=40 + hd)


CHUNKS = {
    "chunks": ((5, 40, 1, 300, 64), (5, 100, 77, 1000, 65), 4, 2),
    "long_past": ((1, 3, 40), (1500, 700, 1300), 8, 1),
    "queries_without_keys": ((40, 17, 100, 33), (17, 0, 99, 1), 6, 2),
    "keys_without_queries": ((0, 20, 0), (9, 50, 140), 2, 2),
    "nothing_but_keys": ((0, 0), (33, 200), 2, 1),
    "nothing_but_queries": ((33, 200), (0, 0), 2, 1),
}


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("name", list(CHUNKS))
def test_lengths_that_differ(name, hd):
    q, kv, heads, kvh = CHUNKS[name]
    _check(q, kv, heads, kvh, hd, seed=50 + hd)


@pytest.mark.parametrize("hd", [64, 128])
def test_peaky_scores_move_the_reference(hd):
    # scores of some tens: the running reference moves in most units
    b = _binding()
    lens = (300, 90)
    dev = _inputs(lens, lens, 4, 2, hd, 60, gain=3.0)
    cu, scale = _cu(lens), hd ** -0.5
    out, lse = b.vfm_cattn_fwd(dev["q"], dev["k"], dev["v"], cu, cu, scale)
    _assert_close(dev, out, lse, None, cu, cu, scale)


def test_more_sequences_than_a_launch_holds():
    rng = np.random.default_rng(3)
    q = [int(x) for x in rng.integers(0, 9, 300)]
    kv = [n + int(x) for n, x in zip(q, rng.integers(0, 40, 300))]
    _check(q, kv, 2, 1, 64, seed=61)


@pytest.mark.parametrize("hd", [64, 128])
def test_parts_of_one_projection(hd):
    """q, k, v and their gradients as parts of one [tokens, heads + 2 kv_heads, head_dim] tensor each: bitwise the same."""
    import torch
    b = _binding()
    lens, heads, kvh = (150, 33, 1, 280), 6, 2
    dev = _inputs(lens, lens, heads, kvh, hd, 62)
    cu, scale = _cu(lens), hd ** -0.5
    out, lse = b.vfm_cattn_fwd(dev["q"], dev["k"], dev["v"], cu, cu, scale)
    grads = b.vfm_cattn_bwd(dev["q"], dev["k"], dev["v"], out, lse, dev["dout"], cu, cu, scale)
    fused = torch.cat((dev["q"], dev["k"], dev["v"]), dim=1)
    parts = (fused[:, :heads], fused[:, heads:heads + kvh], fused[:, heads + kvh:])
    o2, l2 = b.vfm_cattn_fwd(*parts, cu, cu, scale)
    dfused = torch.full_like(fused, float("nan"))
    dparts = (dfused[:, :heads], dfused[:, heads:heads + kvh], dfused[:, heads + kvh:])
    b.vfm_cattn_bwd(*parts, o2, l2, dev["dout"], cu, cu, scale, *dparts)
    assert torch.equal(out, o2) and torch.equal(lse, l2)
    for got, want in zip(dparts, grads):
        assert torch.equal(got, want)


def test_same_bits_every_time_and_whatever_else_is_in_the_pack():
    import torch
    b = _binding()
    lens = (700, 41, 1300, 5)
    dev, out, lse, grads = _check(lens, lens, 4, 2, 128, seed=63)
    cu, scale = _cu(lens), 128 ** -0.5
    for _ in range(2):
        o2, l2 = b.vfm_cattn_fwd(dev["q"], dev["k"], dev["v"], cu, cu, scale)
        g2 = b.vfm_cattn_bwd(dev["q"], dev["k"], dev["v"], o2, l2, dev["dout"], cu, cu, scale)
        assert all(torch.equal(x, y) for x, y in zip((out, lse, *grads), (o2, l2, *g2)))


def test_on_a_stream_of_the_callers_and_in_a_graph():
    import torch
    b = _binding()
    q, kv = (70, 1, 300), (170, 1, 300)
    cq, ck, scale = _cu(q), _cu(kv), 128 ** -0.5
    dev = _inputs(q, kv, 8, 2, 128, 64)
    out, lse = b.vfm_cattn_fwd(dev["q"], dev["k"], dev["v"], cq, ck, scale)
    grads = b.vfm_cattn_bwd(dev["q"], dev["k"], dev["v"], out, lse, dev["dout"], cq, ck, scale)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    o2, l2 = b.vfm_cattn_fwd(dev["q"], dev["k"], dev["v"], cq, ck, scale, stream=side)
    g2 = b.vfm_cattn_bwd(dev["q"], dev["k"], dev["v"], o2, l2, dev["dout"], cq, ck, scale, stream=side)
    side.synchronize()
    assert all(torch.equal(x, y) for x, y in zip((out, lse, *grads), (o2, l2, *g2)))
    ws = torch.empty(max(b.vfm_cattn_bwd_workspace_size(cq, ck, 8, 2, 128), b.vfm_cattn_fwd_workspace_size(cq, ck, 8, 2, 128), 256),
                     dtype=torch.uint8, device="cuda")
    got = [torch.zeros_like(x) for x in (out, lse, *grads)]

    def step():
        b.vfm_cattn_fwd(dev["q"], dev["k"], dev["v"], cq, ck, scale, out=got[0], lse=got[1], workspace=ws)
        b.vfm_cattn_bwd(dev["q"], dev["k"], dev["v"], got[0], got[1], dev["dout"], cq, ck, scale, *got[2:], workspace=ws)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for gain in (1.0, 0.5, 2.0):
        dev["q"].mul_(gain)
        step()
        torch.cuda.synchronize()
        want = [x.clone() for x in got]
        for x in got:
            x.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, want))


def test_gradients_against_differences():
    """The loss sum(out * dout) along random directions of q, k, v, by central differences of the forward in 64 bits' place: the
    kernel's out is bf16, so the difference is taken of the oracle's forward at the kernel's own inputs, and the
    kernel's gradients have to predict it."""
    lens = (37, 80)
    dev, out, lse, grads = _check(lens, lens, 4, 2, 64, seed=65)
    host = {n: U.to_f64(t) for n, t in dev.items()}
    cu, scale = _cu(lens), 64 ** -0.5
    rng = np.random.default_rng(1)
    for n, g in zip(("q", "k", "v"), grads):
        d = rng.standard_normal(host[n].shape)
        f = []
        for step in (1e-4, -1e-4):
            moved = dict(host)
            moved[n] = host[n] + step * d
            f.append(float((orc.cattn_fwd(moved["q"], moved["k"], moved["v"], cu, cu, scale)[0] * host["dout"]).sum()))
        got, size = float((U.to_f64(g) * d).sum()), float(np.linalg.norm(U.to_f64(g)))
        # a direction's slope sums the elements' errors with random signs: the norm's bound, four sigma
        assert abs((f[0] - f[1]) / 2e-4 - got) <= 4 * U.TOL_GRAD_RELRMS * size, n


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("heads", [71, 140])
def test_groups_wider_than_a_tile(heads, hd):
    """One K/V head for more query heads than a row block, or a tile, has rows."""
    _check((9, 1, 70), (40, 1, 70), heads, 1, hd, seed=70 + hd)
