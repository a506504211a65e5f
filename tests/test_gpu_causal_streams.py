"""Causal attention and the 4-bit cache on a stream of the caller's while the current stream still works on memory that it has freed."""
import pytest

from tests.test_gpu_cattn_special import _binding, _cu, _inputs

pytestmark = pytest.mark.gpu


def test_results_do_not_lie_where_the_current_stream_still_writes():
    """Tensors of the results' sizes are freed with writes to them still to come; results of calls on another stream keep their values."""
    import torch
    b = _binding()
    heads, kvh, hd, n = 8, 2, 64, 1500
    cu, scale = _cu((n,)), hd ** -0.5
    dev = _inputs((n,), (n,), heads, kvh, hd, 190)
    cache = [torch.zeros(30, kvh, 64, x, device="cuda", dtype=torch.uint8) for x in (32, 32, 2, 2)]
    pages, lens = torch.arange(30, device="cuda", dtype=torch.int32).view(1, 30), torch.zeros(1, device="cuda", dtype=torch.int32)
    step = _cu((4,))

    def calls(stream):
        out, lse = b.vfm_cattn_fwd(dev["q"], dev["k"], dev["v"], cu, cu, scale, stream=stream)
        grads = b.vfm_cattn_bwd(dev["q"], dev["k"], dev["v"], out, lse, dev["dout"], cu, cu, scale, stream=stream)
        b.vfm_kv4_append(dev["k"], dev["v"], *cache, pages, lens, cu, stream=stream)
        rows = b.vfm_kv4_gather(*cache, pages, cu, stream=stream)
        return (out, lse, *grads, *rows, *b.vfm_kv4_attn(dev["q"][:4], *cache, pages, later, step, scale, stream=stream))

    later = lens + 1000
    want = [t.clone() for t in calls(None)]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(2):
        gone = [torch.empty_like(t) for t in want]
        torch.cuda._sleep(200_000_000)                       # some tenths of a second in front of the writes
        for t in gone:
            t.fill_(7)
        del gone, t
        got = calls(side)
        side.synchronize()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, want))
        del got
