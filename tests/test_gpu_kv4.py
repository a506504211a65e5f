"""GPU tests of the 4-bit key/value cache: rows written and read back exactly as the oracle does, attention over it
against 64 bits.

Bounds of the attention: q, the codes and their factors are exact, P is rounded to bf16 before the second product and
out after it: 5e-3 in the RMS of a tensor, three times that per row (as in test_gpu_cattn.py); lse 1e-3."""
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


class Cache:
    """A cache with scattered pages; its bytes are garbage to begin with (scale bytes 255 among them)."""

    def __init__(self, room, kvh, hd, page, seed=0, spare=2):
        import torch
        rng = np.random.default_rng(seed)
        need = [-(-n // page) for n in room]
        n_pages = sum(need) + spare
        order = rng.permutation(n_pages).astype(np.int32)
        self.table = np.full((len(room), max(max(need), 1)), -1, dtype=np.int32)
        at = 0
        for s, n in enumerate(need):
            self.table[s, :n] = order[at:at + n]
            at += n
        self.page, self.kvh, self.hd = page, kvh, hd
        draw = lambda last: torch.from_numpy(rng.integers(0, 256, (n_pages, kvh, page, last), dtype=np.uint8)).cuda()  # noqa: E731
        self.bufs = [draw(hd // 2), draw(hd // 2), draw(hd // 32), draw(hd // 32)]
        self.bufs[2][..., 0] = 255
        self.bufs[3][..., -1] = 255
        self.pages = torch.from_numpy(self.table).cuda()

    def host(self):
        return [t.cpu().numpy() for t in self.bufs]


def _dev_i32(x):
    import torch
    return torch.tensor([int(v) for v in x], dtype=torch.int32, device="cuda")


def _bits(seed, name, shape, gain=1.0):
    return W.f32_to_bf16_bits(W.normal_f32(seed, name, shape, gain))


def _fill(c, lens, seed, gain=1.0):
    """The first lens[s] places of every sequence, appended in one call."""
    b = _binding()
    total = sum(lens)
    k, v = (U.to_device(_bits(seed, n, (total, c.kvh, c.hd), gain)) for n in ("k", "v"))
    b.vfm_kv4_append(k, v, *c.bufs, c.pages, _dev_i32([0] * len(lens)), _cu(lens))
    return k, v


SPECIALS = np.array([0.0, -0.0, 6.0, -6.0, 6.03125, 3.0, 3.015625, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.25, -5.0, 448.0, 1e-3, 1e-20,
                     -1e-30, 1e-38, 1e-40, 9e-41, 2.0 ** -126, 3e38, -3.3e38, 1e30, 0.2490, 0.2510, 4.96875, 5.03125, 1.0], dtype=np.float32)


@pytest.mark.parametrize("hd,page", [(64, 16), (128, 64)])
def test_rows_are_kept_as_the_format_says(hd, page):
    import torch
    b = _binding()
    lens = (37, 1, 0, 130, 16)
    total, kvh = sum(lens), 3
    c = Cache(lens, kvh, hd, page, seed=1)
    rng = np.random.default_rng(2)
    x = rng.standard_normal((2, total, kvh, hd)).astype(np.float32) * np.exp2(rng.integers(-30, 30, (2, total, kvh, 1)))
    x[0, 3] = 0.0
    x[1, 5:25] = rng.choice(SPECIALS, (20, kvh, hd))
    x[0, 6, 0] = np.tile(SPECIALS, hd // 32)
    for i, s in enumerate((0, 2, 7, 17, 20)):                   # one large value sets a block's scale
        x[0, 7 + i] = 2.0 ** -6 * rng.standard_normal((kvh, hd))
        x[0, 7 + i, :, s] = SPECIALS[6 + i]
    x[1, 30, 1, 5], x[1, 31, 0, 40 % hd], x[0, 32, 2, 0] = np.nan, np.inf, -np.inf
    k, v = (U.to_device(W.f32_to_bf16_bits(y)) for y in x)
    before = c.host()
    b.vfm_kv4_append(k, v, *c.bufs, c.pages, _dev_i32([0] * 5), _cu(lens))
    after = c.host()
    want = [y.copy() for y in before]
    cu = _cu(lens)
    for t, codes, scales in ((k, 0, 2), (v, 1, 3)):
        wc, ws = orc.kv4_encode(U.to_f64(t))
        for s in range(len(lens)):
            for i in range(lens[s]):
                p = c.table[s, i // page]
                want[codes][p, :, i % page] = wc[cu[s] + i]
                want[scales][p, :, i % page] = ws[cu[s] + i]
    for i, (got, w) in enumerate(zip(after, want)):
        # every byte of the cache: rows as the oracle writes them, everything else left alone.  (A zero may have either sign.)
        if i < 2:
            low = lambda y: np.where(y & 7, y, 0)  # noqa: E731
            assert np.array_equal(low(got & 15), low(w & 15)) and np.array_equal(low(got >> 4), low(w >> 4)), i
        else:
            assert np.array_equal(got, w), i
    gk, gv = b.vfm_kv4_gather(*c.bufs, c.pages, cu)
    for t, codes, scales in ((gk, 0, 2), (gv, 1, 3)):
        ref = np.concatenate([orc.kv4_rows(after[codes], after[scales], c.table[s], lens[s])[0] for s in range(len(lens))])
        with np.errstate(invalid="ignore"):
            assert np.array_equal(U.to_f64(t), ref, equal_nan=True)
    assert torch.isnan(gv[30, 1, :32]).all()


@pytest.mark.parametrize("hd,page", [(64, 32), (128, 16)])
def test_places_that_are_not_there(hd, page):
    """Idle slots, entries that name no page, places past the table: neither written nor read, gathered as zeros."""
    import torch
    b = _binding()
    kvh, heads = 2, 6
    c = Cache((40, 100, 70, 20), kvh, hd, page, seed=3)
    c.table[1, 1] = -5
    c.table[2, 0] = c.bufs[0].shape[0]
    c.pages.copy_(torch.from_numpy(c.table))
    lens, new = (30, 2, -1, c.table.shape[1] * page - 2), (3, 60, 4, 5)
    cu = _cu(new)
    before = c.host()
    k, v = (U.to_device(_bits(4, n, (sum(new), kvh, hd))) for n in ("k", "v"))
    b.vfm_kv4_append(k, v, *c.bufs, c.pages, _dev_i32(lens), cu)
    after = c.host()
    written = np.zeros(before[0].shape[::2], dtype=bool)        # [pages, places]
    for s in range(4):
        for i in range(new[s]):
            pos = lens[s] + i
            if lens[s] >= 0 and pos // page < c.table.shape[1] and 0 <= c.table[s, pos // page] < written.shape[0]:
                written[c.table[s, pos // page], pos % page] = True
    for x, y in zip(before, after):
        assert np.array_equal(x.swapaxes(1, 2)[~written], y.swapaxes(1, 2)[~written])
    # make all that is there finite, then look at it
    for t in c.bufs[2:]:
        t.copy_(torch.randint(124, 129, t.shape, dtype=torch.uint8, device="cuda"))
    take = (50, 90, 33, 20)
    gk, _ = b.vfm_kv4_gather(*c.bufs, c.pages, _cu(take))
    host = c.host()
    assert np.array_equal(U.to_f64(gk), np.concatenate([orc.kv4_rows(host[0], host[2], c.table[s], take[s])[0] for s in range(4)]))
    q = U.to_device(_bits(5, "q", (sum(new), heads, hd)))
    _attend(c, q, lens, cu)


def _attend(c, q, lens, cu, **more):
    b = _binding()
    scale = c.hd ** -0.5
    out, lse = b.vfm_kv4_attn(q, *c.bufs, c.pages, _dev_i32(lens), cu, scale, **more)
    host = c.host()
    o_ref, l_ref = orc.kv4_attn(U.to_f64(q), host[0], host[1], host[2], host[3], c.table, np.asarray(lens), cu, scale)
    o, l = U.to_f64(out), U.to_f64(lse)
    assert np.array_equal(np.isnan(l), np.isnan(l_ref)) and np.array_equal(np.isnan(o), np.isnan(o_ref))
    assert np.array_equal(np.isneginf(l), np.isneginf(l_ref))
    some = np.isfinite(l_ref)
    assert U.max_abs(l[some], l_ref[some]) <= U.TOL_LSE_MAXABS
    assert not o[np.isneginf(l_ref).T].any()
    o, o_ref = o[some.T], o_ref[some.T]
    assert U.rel_rms(o, o_ref) <= U.TOL_OUT_RELRMS
    U.assert_rows_close("out", o, o_ref, U.TOL_OUT_RELRMS)
    return out, lse


ATTN = {   # tokens before, new tokens, heads, kv heads, page
    "first_token": ((0,), (1,), 2, 1, 16),
    "single_tokens": ((0, 1, 14, 15, 16, 31, 127, 128, 300), (1,) * 9, 4, 2, 16),
    "sixteen_rows": ((200, 33), (1, 1), 16, 1, 32),
    "seventeen_rows": ((130, 5), (1, 17), 2, 2, 64),
    "thirty_two_rows": ((77, 500, 0), (8, 3, 8), 4, 1, 16),
    "odd_group": ((90, 260), (7, 2), 14, 2, 128),
    "many_rows": ((100, 0, 3), (70, 33, 1), 6, 2, 16),
    "nothing_new": ((50, 60, 70), (0, 2, 0), 4, 4, 16),
    "pages_beyond": ((1000, 20), (1, 2), 8, 8, 256),
}


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("name", list(ATTN))
def test_attention_over_the_cache(name, hd):
    lens, new, heads, kvh, page = ATTN[name]
    have = [a + b for a, b in zip(lens, new)]
    c = Cache(have, kvh, hd, page, seed=6)      # what lies behind a sequence's end is garbage
    _fill(c, have, 7)
    _attend(c, U.to_device(_bits(8, "q", (sum(new), heads, hd))), lens, _cu(new))


@pytest.mark.parametrize("hd", [64, 128])
def test_peaky_scores_and_split_sequences(hd):
    # long pasts against few units: every unit is cut into pieces, whose references differ by tens
    lens, new = (6000, 40, 2500), (1, 2, 1)
    have = [a + b for a, b in zip(lens, new)]
    c = Cache(have, 1, hd, 64, seed=9)
    _fill(c, have, 10, gain=3.0)
    q = U.to_device(_bits(11, "q", (4, 4, hd), 3.0))
    out, lse = _attend(c, q, lens, _cu(new))
    import torch
    for _ in range(2):
        o2, l2 = _attend(c, q, lens, _cu(new))
        assert torch.equal(out, o2) and torch.equal(lse, l2)


@pytest.mark.parametrize("new", [1, 6])
def test_a_nan_reaches_only_those_who_see_it(new):
    """A new token's key or value with a NaN: its own query and those behind it are NaN, those before it and the other K/V
    heads and sequences are not."""
    b = _binding()
    lens, kvh, heads, hd = (45, 45), 2, 6, 128
    c = Cache((60, 60), kvh, hd, 16, seed=12)
    _fill(c, [45, 45], 13)
    k, v = (U.to_device(_bits(14, n, (2 * new, kvh, hd))) for n in ("k", "v"))
    at = new // 2
    k[at, 0, 100] = float("nan")
    v[new + at, 1, 3] = float("inf")
    cu = _cu((new, new))
    b.vfm_kv4_append(k, v, *c.bufs, c.pages, _dev_i32(lens), cu)
    out, _ = _attend(c, U.to_device(_bits(15, "q", (2 * new, heads, hd))), lens, cu)
    bad = U.to_f64(out)
    bad = np.isnan(bad).all(axis=-1)
    want = np.zeros((2 * new, heads), dtype=bool)
    want[at:new, :3] = True
    want[new + at:, 3:] = True
    assert np.array_equal(bad, want)


def test_more_sequences_than_a_launch_holds():
    rng = np.random.default_rng(4)
    lens = [int(x) for x in rng.integers(-1, 60, 300)]
    new = [int(x) for x in rng.integers(0, 3, 300)]
    c = Cache([max(0, a) + b for a, b in zip(lens, new)], 1, 64, 16, seed=16)
    _fill(c, [max(0, a) + b if a >= 0 else 0 for a, b in zip(lens, new)], 17)
    _attend(c, U.to_device(_bits(18, "q", (sum(new), 2, 64))), lens, _cu(new))


def test_query_part_of_a_projection_and_a_workspace_of_the_callers():
    import torch
    b = _binding()
    lens, new = (100, 7), (1, 1)
    c = Cache((101, 8), 2, 64, 16, seed=19)
    k, v = _fill(c, (101, 8), 20)
    wide = U.to_device(_bits(21, "q", (2, 9, 64)))
    cu = _cu(new)
    size = b.vfm_kv4_attn_workspace_size(cu, 4, 2, 64)
    assert size % 256 == 0
    ws = torch.full((size,), 255, dtype=torch.uint8, device="cuda")      # (as floats: NaN)
    got = _attend(c, wide[:, 2:6], lens, cu, workspace=ws)
    want = b.vfm_kv4_attn(wide[:, 2:6].contiguous(), *c.bufs, c.pages, _dev_i32(lens), cu, 64 ** -0.5)
    assert all(torch.equal(x, y) for x, y in zip(got, want))
    # keys and values of a projection's output
    fused = torch.cat((k, v), dim=1)
    before = [t.clone() for t in c.bufs]
    for t in c.bufs:
        t.zero_()
    b.vfm_kv4_append(fused[:, :2], fused[:, 2:], *c.bufs, c.pages, _dev_i32((0, 0)), _cu((101, 8)))
    g1 = b.vfm_kv4_gather(*c.bufs, c.pages, _cu((101, 8)))
    g0 = b.vfm_kv4_gather(*before, c.pages, _cu((101, 8)))
    assert all(torch.equal(x, y) for x, y in zip(g0, g1))


def test_a_captured_step_serves_a_growing_cache():
    """One graph of append and attention, replayed while the lengths grow past page ends and a slot falls idle; two
    graphs share a workspace."""
    import torch
    b = _binding()
    kvh, heads, hd, page = 2, 8, 128, 16
    start = [14, 0, 130, 31]
    c = Cache([n + 40 for n in start], kvh, hd, page, seed=22)
    _fill(c, start, 23)
    cu, scale = _cu((1, 1, 1, 1)), hd ** -0.5
    lens = _dev_i32(start)
    q, k, v = (torch.zeros((4, h, hd), dtype=torch.bfloat16, device="cuda") for h in (heads, kvh, kvh))
    out, lse = torch.zeros_like(q), torch.zeros((heads, 4), dtype=torch.float32, device="cuda")
    ws = torch.zeros(b.vfm_kv4_attn_workspace_size(cu, heads, kvh, hd), dtype=torch.uint8, device="cuda")

    def step():
        b.vfm_kv4_append(k, v, *c.bufs, c.pages, lens, cu)
        b.vfm_kv4_attn(q, *c.bufs, c.pages, lens, cu, scale, out=out, lse=lse, workspace=ws)

    step()
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            step()
    have = list(start)
    for n in range(36):
        for t, h, name in ((q, heads, "q"), (k, kvh, "k"), (v, kvh, "v")):
            t.copy_(U.to_device(_bits(100 + n, name, (4, h, hd))))
        if n == 20:
            lens[1] = -1
            have[1] = -1
        graphs[n % 2].replay()
        torch.cuda.synchronize()
        if n % 7 == 0 or n >= 34:
            got = out.clone(), lse.clone()
            want = _attend(c, q, have, cu)
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        lens += (lens >= 0).to(torch.int32)
        have = [x + 1 if x >= 0 else x for x in have]


def test_on_a_stream_of_the_callers():
    import torch
    b = _binding()
    lens, new = (90, 1200), (2, 1)
    have = [a + b_ for a, b_ in zip(lens, new)]
    c = Cache(have, 2, 128, 64, seed=24)
    q = U.to_device(_bits(25, "q", (3, 8, 128)))
    k, v = (U.to_device(_bits(26, n, (sum(have), 2, 128))) for n in ("k", "v"))
    zero, n = _dev_i32((0, 0)), _dev_i32(lens)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    b.vfm_kv4_append(k, v, *c.bufs, c.pages, zero, _cu(have), stream=side)
    out, lse = b.vfm_kv4_attn(q, *c.bufs, c.pages, n, _cu(new), 128 ** -0.5, stream=side)
    gk, _ = b.vfm_kv4_gather(*c.bufs, c.pages, _cu(have), stream=side)
    side.synchronize()
    want = _attend(c, q, lens, _cu(new))
    assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
    assert torch.equal(gk, b.vfm_kv4_gather(*c.bufs, c.pages, _cu(have))[0])


@pytest.mark.parametrize("hd", [64, 128])
def test_a_prompt_in_chunks_then_tokens(hd):
    """The calls as they are used: a prompt goes through the cache chunk by chunk (append, gather, causal attention of the chunk
    against all before it), then single tokens attend to the cache.  A chunk's last token and a single token that sees the
    same keys agree, and every step matches 64 bits on what the cache holds."""
    import torch
    b = _binding()
    kvh, heads, page, scale = 2, 8, 32, hd ** -0.5
    prompts = [(70, 5), (64, 40), (1, 33)]            # chunks of two sequences
    total = [sum(x) for x in zip(*prompts)]
    c = Cache([n + 3 for n in total], kvh, hd, page, seed=27)
    have = [0, 0]
    for n, new in enumerate([*prompts, (1, 1), (1, 1), (1, 1)]):
        cu = _cu(new)
        q, k, v = (U.to_device(_bits(30 + n, name, (sum(new), h, hd))) for name, h in (("q", heads), ("k", kvh), ("v", kvh)))
        b.vfm_kv4_append(k, v, *c.bufs, c.pages, _dev_i32(have), cu)
        upto = _cu([a + b_ for a, b_ in zip(have, new)])
        gk, gv = b.vfm_kv4_gather(*c.bufs, c.pages, upto)
        out, lse = b.vfm_cattn_fwd(q, gk, gv, cu, upto, scale)
        o2, l2 = _attend(c, q, have, cu)
        # the same sums in another order, rounded once: half a step of bf16 each
        assert U.max_abs(U.to_f64(lse), U.to_f64(l2)) <= U.TOL_LSE_MAXABS
        assert U.rel_rms(U.to_f64(out), U.to_f64(o2)) <= U.TOL_OUT_RELRMS
        have = [a + b_ for a, b_ in zip(have, new)]
    assert torch.isfinite(out).all()


@pytest.mark.parametrize("hd", [64, 128])
def test_lengths_far_past_the_table(hd):
    """A sequence whose length no table holds: its new tokens see the whole table and are not kept themselves."""
    b = _binding()
    lens, new, kvh = (2 ** 31 - 1, 2 ** 31 - 2, 60, 2 ** 30), (3, 1, 2, 40), 2
    c = Cache((60, 20, 64, 33), kvh, hd, 16, seed=30)
    room = c.table.shape[1] * 16
    for s, n in enumerate((4, 2, 4, 3)):            # (tables shorter than the widest one end in -1)
        assert (c.table[s] >= 0).sum() == n and room == 64
    _fill(c, (60, 20, 62, 33), 31)
    for t in c.bufs[2:]:
        t.clamp_(max=130)
    before = [t.clone() for t in c.bufs]
    k, v = (U.to_device(_bits(32, n, (sum(new), kvh, hd))) for n in ("k", "v"))
    b.vfm_kv4_append(k, v, *c.bufs, c.pages, _dev_i32(lens), _cu(new))
    changed = np.zeros((before[0].shape[0], 16), dtype=bool)
    for t, old in zip(c.bufs, before):
        changed |= (t != old).any(dim=3).any(dim=1).cpu().numpy()
    want = np.zeros_like(changed)
    want[c.table[2, 60 // 16], [60 % 16, 61 % 16]] = True
    assert np.array_equal(changed, want)
    _attend(c, U.to_device(_bits(33, "q", (sum(new), 4, hd))), lens, _cu(new))


@pytest.mark.parametrize("hd", [64, 128])
def test_sequences_that_share_pages(hd):
    """Two sequences with one prompt's pages in common and ends of their own; one call's table, two streams in turn."""
    import torch
    b = _binding()
    c = Cache((96, 40, 8), 2, hd, 32, seed=34)
    _fill(c, (96, 40, 8), 35)
    for t in c.bufs[2:]:
        t.clamp_(max=130)
    c.table[1, :3] = c.table[0, :3]
    c.table[1, 2] = c.table[2, 0]                   # 64 places of the first one's, then the third's page
    c.pages.copy_(torch.from_numpy(c.table))
    lens, new = (90, 66, 5), (2, 4, 1)
    q = U.to_device(_bits(36, "q", (sum(new), 6, hd)))
    out, lse = _attend(c, q, lens, _cu(new))
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = b.vfm_kv4_attn(q, *c.bufs, c.pages, _dev_i32(lens), _cu(new), hd ** -0.5, stream=side)
    side.synchronize()
    assert torch.equal(out, got[0]) and torch.equal(lse, got[1])


def test_a_cache_past_four_gib():
    """Pages at the far end of a cache whose codes take 5 GiB a tensor: the same bytes and results as in a small one."""
    import torch
    b = _binding()
    hd, kvh, page, n_pages = 128, 8, 64, 163840
    lens, new = (150, 63), (2, 1)
    small = Cache((152, 64), kvh, hd, page, seed=40, spare=0)
    _fill(small, (152, 64), 41)
    big = [torch.empty((n_pages, kvh, page, n), dtype=torch.uint8, device="cuda") for n in (64, 64, 4, 4)]
    assert big[0].numel() == 5 << 30
    far = Cache((152, 64), kvh, hd, page, seed=40, spare=0)
    used = int(small.table.max()) + 1
    far.table = np.where(small.table >= 0, n_pages - used + small.table, -1).astype(np.int32)
    far.pages.copy_(torch.from_numpy(far.table))
    far.bufs = big
    _fill(far, (152, 64), 41)
    for x, y in zip(b.vfm_kv4_gather(*small.bufs, small.pages, _cu((152, 64))), b.vfm_kv4_gather(*far.bufs, far.pages, _cu((152, 64)))):
        assert torch.equal(x, y)
    q = U.to_device(_bits(42, "q", (3, 16, hd)))
    got = b.vfm_kv4_attn(q, *far.bufs, far.pages, _dev_i32(lens), _cu(new), hd ** -0.5)
    for t in small.bufs[2:]:
        t.clamp_(max=254)
    want = _attend(small, q, lens, _cu(new))
    # (places of the last pages past the sequences' ends differ: nobody sees them)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("hd", [64, 128])
def test_groups_wider_than_a_row_block(hd):
    lens, new = (130, 0, 700), (1, 2, 3)
    have = [a + b for a, b in zip(lens, new)]
    c = Cache(have, 2, hd, 32, seed=43)
    _fill(c, have, 44)
    _attend(c, U.to_device(_bits(45, "q", (sum(new), 140, hd))), lens, _cu(new))


@pytest.mark.parametrize("hd", [64, 128])
def test_a_cache_without_pages(hd):
    import torch
    pkg = _binding()
    # no memory at all behind the table's entries: nothing is written, zeros are read, no token sees anything
    kvh, heads, page, cu = 2, 8, 16, np.array([0, 1, 6], np.int32)
    cache = [torch.empty((0, kvh, page, n), dtype=torch.uint8, device="cuda") for n in (hd // 2, hd // 2, hd // 32, hd // 32)]
    pages = torch.zeros((2, 40), dtype=torch.int32, device="cuda")
    lens = torch.tensor([600, 3], dtype=torch.int32, device="cuda")
    kv = torch.ones((6, kvh, hd), dtype=torch.bfloat16, device="cuda")
    q = torch.ones((6, heads, hd), dtype=torch.bfloat16, device="cuda")
    pkg.vfm_kv4_append(kv, kv, *cache, pages, lens, cu)
    k, v = pkg.vfm_kv4_gather(*cache, pages, cu, torch.ones_like(kv), torch.ones_like(kv))
    assert not k.any() and not v.any()
    out, lse = pkg.vfm_kv4_attn(q, *cache, pages, lens, cu, hd ** -0.5, torch.ones_like(q))
    assert not out.any() and bool((lse == -float("inf")).all())
