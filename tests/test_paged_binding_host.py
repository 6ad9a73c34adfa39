"""What the binding of the paged calls refuses before it touches a device (runs without a GPU)."""
import pytest
import torch

import paper_2604_05438_b200 as T
from paper_2604_05438_b200.build import build_library


@pytest.fixture(scope="module")
def kv():
    build_library()
    k = torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16)
    return T.PagedKVCache(k, k.clone(), torch.zeros(1, 4, dtype=torch.int32), [20], [0, 1], 4, torch.zeros(4, 2, 2, 64, dtype=torch.bfloat16))


Q, WS = torch.zeros(1, 4, 64, dtype=torch.bfloat16), torch.zeros(1024, dtype=torch.uint8)


@pytest.mark.parametrize("scale", [0.0, -1.0, float("nan"), float("inf"), 1e39, 1e-46, 1e-300])
def test_scales_that_32_bits_do_not_hold(kv, scale):
    # (1e-46 is 0 in 32 bits, which would stand for 1 / sqrt(head_dim))
    with pytest.raises(ValueError, match="scale"):
        T.paged_attention(kv, Q, Q.clone(), None, scale, T.FLAG_NONE, WS)
    with pytest.raises(ValueError, match="scale"):
        T.paged_block_attention(kv, T.PageSelection(1, 1, 2), Q, Q.clone(), None, None, scale, WS)


@pytest.mark.parametrize("scale", [None, 1e-40, 1, 3e38])
def test_scales_that_are_taken(kv, scale):
    with pytest.raises(ValueError, match="device"):                    # the next check
        T.paged_attention(kv, Q, Q.clone(), None, scale, T.FLAG_NONE, WS)


@pytest.mark.parametrize("flags", [1 << 32, (1 << 32) + 2, 1 << 40])
def test_flags_beyond_32_bits(kv, flags):
    with pytest.raises(ValueError, match="flags"):
        T.paged_attention(kv, Q, Q.clone(), None, None, flags, WS)


@pytest.mark.parametrize("flags", [-1, 1 << 70])
def test_flags_that_are_no_unsigned_word(kv, flags):
    with pytest.raises(OverflowError):
        T.paged_attention(kv, Q, Q.clone(), None, None, flags, WS)


def test_selections_out_of_range(kv):
    for bad in ((1 << 25, 1, 1), (1, -2, 1), (1, 1, 1 << 62)):
        with pytest.raises(ValueError, match="selection"):
            T.paged_block_attention(kv, T.PageSelection(*bad), Q, Q.clone(), None, None, None, WS)


def test_the_longest_sequence():
    # 2^30 rows: beyond it a length and a chunk of it no longer add up within 31 bits on the device (a table may repeat pages,
    # so that such a cache need not be large)
    import test_paged_host as H
    lib = T.load_library()
    for d, page in ((64, 16), (128, 128)):
        for rows, status in ((1 << 30, -3), ((1 << 30) + 1, -1), ((1 << 31) - 1025, -1)):
            desc = H.Desc(lens=((1, rows), (500, rows)), d=d, ps=page, strides=(2 * page * d, page * d, d), max_pages=(1 << 31) // page)
            assert H._attend(lib, desc, ws=0) == status, (rows, lib.tkphi_last_error())
            if status == -1:
                assert H._append(lib, desc, rot_dim=d, inv_freq=0) == -1 and b"kv_lens" in lib.tkphi_last_error()


def test_pairs_without_a_truth_value(kv):
    import numpy as np
    k = torch.zeros(1, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="truth value"):
        T.paged_append(kv, k, k, T.RotaryMap(torch.zeros(8), np.array([True, False])))
