"""Pins of the oracle's causal attention with grouped heads and of its 4-bit cache: loops over single numbers, PyTorch's
autograd in 64 bits, differences, and the format's own tables."""
import math

import numpy as np
import pytest

from oracle import vfm_oracle as orc

CASES = [   # queries, keys, heads, kv heads
    ((5, 3), (5, 3), 2, 2),
    ((4, 1, 2), (7, 1, 5), 6, 2),
    ((5, 2, 3), (3, 0, 3), 3, 1),
]


def _draw(q, kv, heads, kvh, d=6, seed=0):
    rng = np.random.default_rng(seed)
    cq, ck = np.concatenate([[0], np.cumsum(q)]), np.concatenate([[0], np.cumsum(kv)])
    return (rng.standard_normal((cq[-1], heads, d)), rng.standard_normal((ck[-1], kvh, d)), rng.standard_normal((ck[-1], kvh, d)),
            rng.standard_normal((cq[-1], heads, d)), cq, ck)


@pytest.mark.parametrize("q,kv,heads,kvh", CASES)
def test_forward_is_the_sum_written_out(q, kv, heads, kvh):
    Q, K, V, _, cq, ck = _draw(q, kv, heads, kvh)
    out, lse = orc.cattn_fwd(Q, K, V, cq, ck, 0.4)
    for s in range(len(q)):
        for i in range(q[s]):
            for h in range(heads):
                n = h // (heads // kvh)
                w = [math.exp(0.4 * sum(Q[cq[s] + i, h, x] * K[ck[s] + j, n, x] for x in range(6)))
                     for j in range(kv[s]) if j <= i + kv[s] - q[s]]
                got = out[cq[s] + i, h]
                if not w:
                    assert not got.any() and lse[h, cq[s] + i] == -np.inf
                    continue
                want = sum(w[j] / sum(w) * V[ck[s] + j, n] for j in range(len(w)))
                assert np.allclose(got, want, atol=1e-13) and abs(lse[h, cq[s] + i] - math.log(sum(w))) < 1e-12


@pytest.mark.parametrize("q,kv,heads,kvh", CASES)
def test_gradients_are_autograds(q, kv, heads, kvh):
    import torch
    Q, K, V, dO, cq, ck = _draw(q, kv, heads, kvh, seed=1)
    t = [torch.tensor(x, requires_grad=True) for x in (Q, K, V)]
    total = 0.0
    for s in range(len(q)):
        a, b, c, d = cq[s], cq[s + 1], ck[s], ck[s + 1]
        first = max(0, q[s] - kv[s])        # queries before it see nothing
        if first >= q[s]:
            continue
        for h in range(heads):
            n = h // (heads // kvh)
            S = 0.3 * (t[0][a + first:b, h] @ t[1][c:d, n].T)
            S = S.masked_fill(~torch.ones(q[s], kv[s], dtype=torch.bool).tril(kv[s] - q[s])[first:], -math.inf)
            total = total + (torch.softmax(S, 1) @ t[2][c:d, n] * torch.tensor(dO[a + first:b, h])).sum()
    total.backward()
    for got, x in zip(orc.cattn_bwd(Q, K, V, dO, cq, ck, 0.3), t):
        want = np.zeros(x.shape) if x.grad is None else x.grad.numpy()
        assert np.allclose(got, want, atol=1e-12)


def test_gradients_against_differences():
    Q, K, V, dO, cq, ck = _draw((4, 2), (6, 2), 4, 2, d=4, seed=2)
    grads = orc.cattn_bwd(Q, K, V, dO, cq, ck, 0.5)
    for n, x in enumerate((Q, K, V)):
        for at in np.ndindex(x.shape):
            keep = x[at]
            f = []
            for step in (1e-6, -1e-6):
                x[at] = keep + step
                f.append((orc.cattn_fwd(Q, K, V, cq, ck, 0.5)[0] * dO).sum())
            x[at] = keep
            assert abs((f[0] - f[1]) / 2e-6 - grads[n][at]) < 1e-7


def test_last_query_of_equal_heads_is_cross_attention():
    Q, K, V, _, _, ck = _draw((1,), (9,), 3, 3, seed=3)
    out, lse = orc.cattn_fwd(Q, K, V, [0, 1], ck, 0.7)
    want, l = orc.xattn_fwd(Q, K, V, [0, 1], ck, 0.7)
    assert np.allclose(out, want, atol=1e-14) and np.allclose(lse, l, atol=1e-14)


# ---------------------------------------------------------------- 4 bits
def test_every_code_reads_as_its_fields_say():
    codes = np.arange(16, dtype=np.uint8).reshape(1, 16) | (np.arange(16, dtype=np.uint8).reshape(1, 16) << 4)
    got = orc.kv4_decode(codes, np.array([[128]], dtype=np.uint8))[0]
    for c in range(16):
        field, half = (c >> 1) & 3, c & 1
        want = 0.5 * half if field == 0 else 2.0 ** (field - 1) * (1 + 0.5 * half)
        assert got[2 * c] == got[2 * c + 1] == (-want if c & 8 else want) * 2.0


@pytest.mark.parametrize("top,byte", [(0.0, 127), (6.0, 127), (6.0625, 128), (3.0, 126), (3.03125, 127), (1.0, 125), (448.0, 134),
                                      (2.0 ** -126, 7), (3.0e38, 252), (2.0 ** 125 * 6, 252), (6 * 2.0 ** -120, 7)])
def test_scale_is_the_largest_that_keeps_the_block(top, byte):
    x = np.zeros((1, 32))
    x[0, 5] = -top
    codes, scales = orc.kv4_encode(x)
    assert scales[0, 0] == byte
    back = orc.kv4_decode(codes, scales)[0, 5]
    assert abs(back) <= 6 * 2.0 ** (byte - 127)
    if top and 7 < byte < 252:
        assert abs(back + top) <= 0.25 * top and top * 2.0 ** (128 - byte) > 6


def test_nearest_value_ties_to_the_even_code():
    x = np.zeros((1, 32))
    x[0, 0] = 6.0
    x[0, 1:9] = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.25]
    x[0, 9:13] = [0.26, 0.74, 5.01, -4.99]
    got = orc.kv4_decode(*orc.kv4_encode(x))[0]
    assert got[1:13].tolist() == [0.0, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0, 0.0, 0.5, 0.5, 6.0, -4.0]
    assert np.signbit(got[8])


def test_a_block_with_a_nan_or_an_infinity_is_nan_alone():
    x = np.ones((1, 64))
    for bad in (np.nan, np.inf, -np.inf):
        x[0, 3] = bad
        codes, scales = orc.kv4_encode(x)
        assert scales.tolist() == [[255, 125]] and not codes[0, :16].any()
        back = orc.kv4_decode(codes, scales)[0]
        assert np.isnan(back[:32]).all() and (back[32:] == 1).all()


def test_cache_attention_is_causal_attention_on_the_values():
    rng = np.random.default_rng(5)
    n_pages, kvh, page, D, heads = 7, 2, 4, 32, 6
    k4, v4 = (rng.integers(0, 256, (n_pages, kvh, page, D // 2), dtype=np.uint8) for _ in range(2))
    ks, vs = (rng.integers(124, 128, (n_pages, kvh, page, 1), dtype=np.uint8) for _ in range(2))
    pages = np.array([[3, 0, 6], [5, 2, 0]])
    lens, cu = np.array([7, 3]), [0, 2, 4]
    q = rng.standard_normal((4, heads, D))
    out, lse = orc.kv4_attn(q, k4, v4, ks, vs, pages, lens, cu, 0.2)
    K = np.concatenate([orc.kv4_rows(k4, ks, pages[s], lens[s] + 2)[0] for s in range(2)])
    V = np.concatenate([orc.kv4_rows(v4, vs, pages[s], lens[s] + 2)[0] for s in range(2)])
    want, l = orc.cattn_fwd(q, K, V, cu, [0, 9, 14], 0.2)
    assert np.allclose(out, want, atol=1e-13) and np.allclose(lse, l, atol=1e-13)
