"""The 4-bit cache over the whole range of bf16: which factors are written, and that every value that they stand for is a bf16."""
import numpy as np
import pytest

from oracle import vfm_oracle as orc
from tests import parity_utils as U
from tests.test_gpu_cattn_special import _binding, _cu

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hd", [64, 128])
def test_factors_keep_to_the_documented_range_and_values_to_bf16(hd):
    """Blocks whose largest magnitude runs through every exponent of bf16, subnormal ones and the largest finite one among them."""
    import torch
    b = _binding()
    kvh, page = 2, 64
    tops = np.concatenate([np.arange(0, 255, dtype=np.uint16) << 7, (np.arange(0, 255, dtype=np.uint16) << 7) | 0x41,
                           np.array([1, 2, 0x40, 0x7f, 0x7f7f], dtype=np.uint16)])
    n = len(tops)
    rng = np.random.default_rng(hd)
    shrink = rng.integers(0, 4, (n, kvh, hd)).astype(np.uint16) << 7
    bits = np.where(tops[:, None, None] >= 4 << 7, tops[:, None, None] - shrink, tops[:, None, None] >> rng.integers(0, 3, (n, kvh, hd)).astype(np.uint16))
    bits[..., ::32] = tops[:, None, None]
    bits = (bits | (rng.integers(0, 2, bits.shape).astype(np.uint16) << 15)).astype(np.uint16)
    rows = U.to_device(bits)
    pages = (n + page - 1) // page
    cache = [torch.zeros(pages, kvh, page, x, device="cuda", dtype=torch.uint8) for x in (hd // 2, hd // 2, hd // 32, hd // 32)]
    table = torch.arange(pages, device="cuda", dtype=torch.int32).view(1, pages)
    lens = torch.zeros(1, device="cuda", dtype=torch.int32)
    b.vfm_kv4_append(rows, rows, *cache, table, lens, _cu((n,)))
    back, _ = b.vfm_kv4_gather(*cache, table, _cu((n,)))
    codes, scales = orc.kv4_encode(U.bits_to_f64(bits))
    written = cache[2].cpu().numpy().transpose(0, 2, 1, 3).reshape(pages * page, kvh, hd // 32)[:n]
    assert np.array_equal(written, scales)
    assert written.min() == 7 and written.max() == 252
    want = orc.kv4_decode(codes, scales)
    assert np.array_equal(U.to_f64(back), want) and np.isfinite(want).all()
