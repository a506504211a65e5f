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
