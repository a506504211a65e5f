"""Refusals of causal attention and of the 4-bit cache, in C and in Python: before anything is launched, so no GPU is needed."""
import ctypes
import os

import numpy as np
import pytest
import torch

from paper_2503_12964_amd import binding as B

FAKE, ODD = 0x10000, 0x10008       # never dereferenced
NULL, SHAPE, CU, DTYPE, WORKSPACE, ALIGN, STRIDE, PAGE = 1, 2, 3, 6, 7, 9, 11, 12


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.LIB_PATH):
        from paper_2503_12964_amd.build import build_lib
        build_lib(verbose=False)
    return B.load_library()


def _p(a):
    return np.ascontiguousarray(a, dtype=np.int32).ctypes.data_as(ctypes.POINTER(ctypes.c_int32))


def _fwd(lib, **change):
    a = dict(q=FAKE, qs=512, k=FAKE, ks=256, v=FAKE, vs=256, cq=[0, 8], ck=[0, 8], n=1, tq=8, tk=8, H=4, Hk=2, D=128, scale=0.1,
             out=FAKE, lse=FAKE, ws=None, wsb=0, dt=0)
    a.update(change)
    cq, ck = _p(a["cq"]), _p(a["ck"])
    return lib.vfm_cattn_fwd(a["q"], a["qs"], a["k"], a["ks"], a["v"], a["vs"], cq, ck, a["n"], a["tq"], a["tk"], a["H"], a["Hk"],
                             a["D"], a["scale"], a["out"], a["lse"], a["ws"], a["wsb"], a["dt"], None)


def _bwd(lib, **change):
    a = dict(q=FAKE, qs=512, k=FAKE, ks=256, v=FAKE, vs=256, o=FAKE, lse=FAKE, do=FAKE, cq=[0, 8], ck=[0, 8], n=1, tq=8, tk=8, H=4,
             Hk=2, D=128, scale=0.1, dq=FAKE, dqs=512, dk=FAKE, dks=256, dv=FAKE, dvs=256, ws=FAKE, wsb=0, dt=0)
    a.update(change)
    return lib.vfm_cattn_bwd(a["q"], a["qs"], a["k"], a["ks"], a["v"], a["vs"], a["o"], a["lse"], a["do"], _p(a["cq"]), _p(a["ck"]),
                             a["n"], a["tq"], a["tk"], a["H"], a["Hk"], a["D"], a["scale"], a["dq"], a["dqs"], a["dk"], a["dks"],
                             a["dv"], a["dvs"], a["ws"], a["wsb"], a["dt"], None)


BAD = [
    (dict(q=None), NULL), (dict(v=None), NULL), (dict(lse=None), NULL),
    (dict(H=5), SHAPE), (dict(H=0), SHAPE), (dict(Hk=0), SHAPE), (dict(D=96), SHAPE), (dict(tq=-1), SHAPE), (dict(tk=-1), SHAPE),
    (dict(scale=0.0), SHAPE), (dict(scale=float("nan")), SHAPE), (dict(scale=3e38), SHAPE),
    (dict(tq=1 << 26, cq=[0, 1 << 26]), SHAPE),                                          # rows of lse
    (dict(tk=1 << 25, ck=[0, 1 << 25]), SHAPE),                                          # one sequence's keys span 4 GiB and more
    (dict(cq=[0, 7]), CU), (dict(ck=[1, 8]), CU), (dict(cq=[0, 5, 4, 8], ck=[0, 1, 2, 8], n=3), CU),
    (dict(dt=1), DTYPE), (dict(q=ODD), ALIGN), (dict(k=ODD), ALIGN),
    (dict(qs=504), STRIDE), (dict(qs=516), STRIDE), (dict(ks=128), STRIDE), (dict(vs=-256), STRIDE), (dict(vs=1 << 40), STRIDE),
]


@pytest.mark.parametrize("change,status", BAD, ids=str)
def test_causal_forward_and_backward_refuse(lib, change, status):
    assert _fwd(lib, **change) == status
    assert _bwd(lib, **change) == status
    assert b"unknown" not in lib.vfm_strerror(status)


@pytest.mark.parametrize("change,status", [
    (dict(o=None), NULL), (dict(do=None), NULL), (dict(dk=None), NULL), (dict(dqs=8), STRIDE), (dict(dvs=260), STRIDE),
    (dict(dv=ODD), ALIGN), (dict(do=ODD), ALIGN), (dict(), WORKSPACE), (dict(ws=None, wsb=1 << 20), WORKSPACE),
    (dict(ws=0x10010, wsb=1 << 20), WORKSPACE)], ids=str)
def test_causal_backward_refuses(lib, change, status):
    assert _bwd(lib, **change) == status


def test_nothing_to_do_is_not_an_error(lib):
    assert _fwd(lib, tq=0, tk=0, cq=[0, 0], ck=[0, 0], q=None, k=None, v=None, out=None, lse=None) == 0
    assert _bwd(lib, tq=0, tk=0, cq=[0, 0], ck=[0, 0], q=None, k=None, v=None, o=None, lse=None, do=None, dq=None, dk=None, dv=None) == 0
    assert _append(lib, total=0, cu=[0, 0], k=None, v=None) == 0
    assert _attn(lib, total=0, cu=[0, 0], q=None, out=None, lse=None) == 0
    assert B.vfm_cattn_bwd_workspace_size([0, 8], [0, 8], 4, 3, 128) == 0           # sizes that are refused
    assert B.vfm_kv4_attn_workspace_size([0, 8], 4, 3, 128) == 0


def _append(lib, **change):
    a = dict(k=FAKE, ks=256, v=FAKE, vs=256, cu=[0, 3, 8], n=2, total=8, lens=FAKE, pages=FAKE, mp=4, k4=FAKE, v4=FAKE, sk=FAKE, sv=FAKE,
             np_=9, page=16, Hk=2, D=128, dt=0)
    a.update(change)
    return lib.vfm_kv4_append(a["k"], a["ks"], a["v"], a["vs"], _p(a["cu"]), len(a["cu"]) - 1, a["total"], a["lens"], a["pages"], a["mp"],
                              a["k4"], a["v4"], a["sk"], a["sv"], a["np_"], a["page"], a["Hk"], a["D"], a["dt"], None)


def _gather(lib, **change):
    a = dict(k=FAKE, v=FAKE, cu=[0, 3, 8], total=8, pages=FAKE, mp=4, k4=FAKE, v4=FAKE, sk=FAKE, sv=FAKE, np_=9, page=16, Hk=2, D=128, dt=0)
    a.update(change)
    return lib.vfm_kv4_gather(a["k4"], a["v4"], a["sk"], a["sv"], a["np_"], a["page"], a["pages"], a["mp"], _p(a["cu"]), len(a["cu"]) - 1,
                              a["total"], a["Hk"], a["D"], a["k"], a["v"], a["dt"], None)


def _attn(lib, **change):
    a = dict(q=FAKE, qs=512, cu=[0, 3, 8], total=8, lens=FAKE, pages=FAKE, mp=4, k4=FAKE, v4=FAKE, sk=FAKE, sv=FAKE, np_=9, page=16, H=4,
             Hk=2, D=128, scale=0.1, out=FAKE, lse=FAKE, ws=FAKE, wsb=0, dt=0)
    a.update(change)
    return lib.vfm_kv4_attn(a["q"], a["qs"], a["k4"], a["v4"], a["sk"], a["sv"], a["np_"], a["page"], a["pages"], a["mp"], a["lens"],
                            _p(a["cu"]), len(a["cu"]) - 1, a["total"], a["H"], a["Hk"], a["D"], a["scale"], a["out"], a["lse"], a["ws"],
                            a["wsb"], a["dt"], None)


CACHE = [(dict(page=24), PAGE), (dict(page=8), PAGE), (dict(page=1 << 21), PAGE), (dict(page=0), PAGE), (dict(np_=-1), PAGE), (dict(mp=-1), PAGE),
         (dict(k4=None), NULL), (dict(sv=None), NULL), (dict(pages=None), NULL), (dict(D=32), SHAPE), (dict(Hk=0), SHAPE),
         (dict(cu=[0, 3, 7]), CU), (dict(dt=1), DTYPE), (dict(v4=ODD), ALIGN), (dict(pages=0x10001), ALIGN)]


@pytest.mark.parametrize("change,status", CACHE, ids=str)
def test_cache_functions_refuse(lib, change, status):
    assert _append(lib, **change) == status
    assert _gather(lib, **change) == status
    assert _attn(lib, **change) == status


def test_cache_functions_refuse_their_own_arguments(lib):
    assert _append(lib, k=None) == NULL and _append(lib, lens=None) == NULL and _append(lib, ks=255) == STRIDE and _append(lib, v=ODD) == ALIGN
    assert _gather(lib, v=None) == NULL and _gather(lib, k=ODD) == ALIGN
    assert _attn(lib, lens=None) == NULL and _attn(lib, H=3) == SHAPE and _attn(lib, scale=-1.0) == SHAPE and _attn(lib, qs=8) == STRIDE
    assert _attn(lib, total=1 << 21, cu=[0, 1 << 21]) == SHAPE
    assert _attn(lib) == WORKSPACE and _attn(lib, ws=None, wsb=1 << 40) == WORKSPACE and _attn(lib, ws=0x10080, wsb=1 << 40) == WORKSPACE


class _Dev(torch.Tensor):
    """A host tensor that says it lives on a GPU: enough to reach the wrappers' checks of shapes, types and devices."""
    is_cuda = property(lambda self: True)
    where = 0

    def get_device(self):
        return self.where

    @classmethod
    def __torch_function__(cls, func, types, args=(), kwargs=None):
        return super().__torch_function__(func, types, args, kwargs or {})


def _dev(*shape, dtype=torch.bfloat16):
    return torch.zeros(shape, dtype=dtype).as_subclass(_Dev)


def test_wrappers_refuse_what_the_kernels_would_misread(lib, monkeypatch):
    monkeypatch.setattr(B, "_current_device", lambda: 0)
    q, k = _dev(8, 4, 64), _dev(8, 2, 64)
    cu = [0, 8]
    out, lse = _dev(8, 4, 64), _dev(4, 8, dtype=torch.float32)
    call = lambda **c: B.vfm_cattn_fwd(*[c.get(n, d) for n, d in (("q", q), ("k", k), ("v", k))], cu, c.get("ck", cu), 0.1,  # noqa: E731
                                       out=c.get("out", out), lse=c.get("lse", lse), stream=0)
    for bad in (dict(q=_dev(8, 4, 64, dtype=torch.float16)), dict(k=_dev(8, 2, 128)), dict(v=_dev(9, 2, 64)), dict(out=_dev(8, 4, 64, dtype=torch.float32)),
                dict(out=_dev(7, 4, 64)), dict(lse=_dev(8, 4, dtype=torch.float32)), dict(q=torch.zeros(8, 4, 64, dtype=torch.bfloat16)),
                dict(q=_dev(8, 64, 4).transpose(1, 2)), dict(q=_dev(8, 4, 128)[:, :, ::2]), dict(ck=[0, 4, 8]), dict(out=_dev(8, 8, 64)[:, ::2])):
        with pytest.raises(ValueError):
            call(**bad)
    far = _dev(8, 2, 64)
    far.where = 1
    with pytest.raises(ValueError, match="current device"):
        call(k=far)
    with pytest.raises(B.VfmError):          # a head count that the library refuses
        call(k=_dev(8, 3, 64), v=_dev(8, 3, 64))
    cache = [_dev(5, 2, 16, 32, dtype=torch.uint8), _dev(5, 2, 16, 32, dtype=torch.uint8), _dev(5, 2, 16, 2, dtype=torch.uint8), _dev(5, 2, 16, 2, dtype=torch.uint8)]
    pages, lens = _dev(1, 3, dtype=torch.int32), _dev(1, dtype=torch.int32)
    for i, bad in ((0, _dev(5, 2, 16, 32, dtype=torch.int8)), (1, _dev(5, 2, 16, 16, dtype=torch.uint8)), (2, _dev(5, 2, 16, 1, dtype=torch.uint8)),
                   (3, _dev(5, 16, 2, 2, dtype=torch.uint8)), (4, _dev(1, 3, dtype=torch.int64)), (4, _dev(2, 3, dtype=torch.int32)),
                   (5, _dev(1, dtype=torch.int64)), (5, _dev(2, dtype=torch.int32))):
        args = [*cache, pages, lens]
        args[i] = bad
        with pytest.raises(ValueError):
            B.vfm_kv4_append(k, k, *args, cu, stream=0)
        with pytest.raises(ValueError):
            B.vfm_kv4_attn(q, *args, cu, 0.1, out=out, lse=lse, stream=0)
    with pytest.raises(ValueError):
        B.vfm_kv4_append(q, q, *cache, pages, lens, cu, stream=0)        # four heads into a cache of two
    with pytest.raises(ValueError):
        B.vfm_kv4_gather(*cache, pages, cu, k=_dev(7, 2, 64), v=k, stream=0)


def test_more_key_rows_than_a_launch_takes(lib):
    change = dict(tk=1 << 20, ck=[0, 1 << 20], H=512, Hk=512, qs=512 * 128, ks=512 * 128, vs=512 * 128, D=128, tq=8)
    assert _fwd(lib, **change) == SHAPE and _bwd(lib, **change) == SHAPE


def test_a_cut_forward_asks_for_its_workspace(lib):
    """One chunk against a long past is cut: without the workspace that it names it is refused."""
    cq, ck = np.array([0, 64], dtype=np.int32), np.array([0, 30000], dtype=np.int32)
    size = B.vfm_cattn_fwd_workspace_size(cq, ck, 32, 8, 128)
    assert size > 0 and size % 256 == 0
    change = dict(tq=64, cq=cq, tk=30000, ck=ck, H=32, Hk=8, qs=32 * 128, ks=8 * 128, vs=8 * 128)
    for ws, wsb in ((None, 1 << 40), (0x10000, size - 1), (0x10080, 1 << 40)):
        assert _fwd(lib, ws=ws, wsb=wsb, **change) == WORKSPACE
