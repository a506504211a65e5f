"""The Python wrappers of causal attention and of the 4-bit cache: what they check and allocate before the library is called (no GPU)."""
import os

import numpy as np
import pytest

from paper_2503_12964_amd import binding as B


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(B.LIB_PATH):
        from paper_2503_12964_amd.build import build_lib
        build_lib(verbose=False)
    return B.load_library()


@pytest.mark.parametrize("size", [B.vfm_cattn_fwd_workspace_size, B.vfm_cattn_bwd_workspace_size])
@pytest.mark.parametrize("cq,ck", [([0, 5, 8], [0, 8]), ([0, 8], [0, 5, 8]), (np.array([], dtype=np.int32), np.array([], dtype=np.int32)), ([0], [])],
                         ids=str)
def test_workspace_sizes_ask_for_as_many_boundaries_of_keys_as_of_queries(size, cq, ck):
    """The library reads n_seqs + 1 of either: a shorter array would be read past its end."""
    with pytest.raises(ValueError):
        size(cq, ck, 4, 2, 128)


class _Streams:
    """As much of torch as the wrappers allocate with: notes the stream that every tensor is asked for on, and whose end it outlives."""

    def __init__(self):
        import contextlib
        import types
        self.now, self.made, self.uint8, outer = types.SimpleNamespace(cuda_stream=7), [], "uint8", self

        @contextlib.contextmanager
        def stream(s):
            was, outer.now = outer.now, s
            yield
            outer.now = was

        def empty(shape, dtype=None, device=None):
            t = types.SimpleNamespace(numel=lambda: 1, data_ptr=lambda: 0, on=outer.now.cuda_stream, kept_for=[])
            t.record_stream = lambda s: t.kept_for.append(s.cuda_stream)
            outer.made.append(t)
            return t

        self.empty, self.empty_like = empty, lambda like: empty(None)
        self.cuda = types.SimpleNamespace(current_stream=lambda: outer.now, stream=stream,
                                          ExternalStream=lambda x: types.SimpleNamespace(cuda_stream=x))


@pytest.mark.parametrize("stream,on,kept_for", [(None, 7, []), (7, 7, []), (9, 9, [7])])
def test_tensors_come_from_the_memory_of_the_stream_that_the_kernels_run_on(monkeypatch, stream, on, kept_for):
    """The current stream's allocator may hand out what work in front of that stream still uses; another stream would not wait for it."""
    import types
    import torch
    fake = _Streams()
    monkeypatch.setattr(B, "_torch", fake)
    like = types.SimpleNamespace(dtype=torch.bfloat16, shape=(3, 2, 64), device="cuda", is_contiguous=lambda: True)
    for shape in ((3, 2, 64), (5, 2, 64)):
        B._new(shape, torch.bfloat16, like, stream)
    B._workspace(None, lambda: 100, (), like, 0, stream)
    assert [t.on for t in fake.made] == [on] * 3
    assert [t.kept_for for t in fake.made] == [kept_for, kept_for, []]


@pytest.mark.parametrize("tokens", [1, 8, 5000])
@pytest.mark.parametrize("which", ["q", "k", "v"])
def test_the_longest_stride_is_the_documented_one(lib, which, tokens):
    """(tokens + 512) * stride * 2 bytes below 4 GiB, for q, k and v: one step of 8 more is refused.  (What is let through is refused for
    its alignment, which is looked at later: nothing is launched.)"""
    import ctypes
    most = (2 ** 32 - 1) // (2 * (tokens + 512)) // 8 * 8
    cu = (ctypes.c_int32 * 2)(0, tokens)
    odd = 0x10008                                              # never dereferenced
    for stride, status in ((most, 9), (most + 8, 2)):
        s = {n: stride if n == which else 512 for n in "qkv"}
        assert lib.vfm_cattn_fwd(odd, s["q"], odd, s["k"], odd, s["v"], cu, cu, 1, tokens, tokens, 4, 2, 128, 0.1, odd, odd, None, 0, 0, None) == status
        assert lib.vfm_cattn_bwd(odd, s["q"], odd, s["k"], odd, s["v"], odd, odd, odd, cu, cu, 1, tokens, tokens, 4, 2, 128, 0.1, odd, 512, odd, 256,
                                 odd, 256, odd, 1 << 40, 0, None) == status
