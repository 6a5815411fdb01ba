"""Calls of the norm and feed-forward operators that the sizes of test_norm_ops.py and test_ffn_ops.py pass by."""
import ctypes

import pytest
import torch

from paper_2402_14800_b200 import binding, build

DEV = "cuda:0"
gpu = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def lib():
    build.build()
    return binding.load_library()


# ------------------------------------------------------------------------------- no device


@pytest.mark.parametrize("h,f", [(8, 8), (64, 8), (128, 448), (72, 136), (520, 264), (520, 1032), (256, 512), (512, 1032),
                                 (1024, 2048), (2040, 5464), (4096, 14336)])
def test_gradients_launch_deals_each_item_once_and_reads_ahead_only_for_an_item(lib, h, f):
    most = 4096
    items, deal = (ctypes.c_int * most)(), (ctypes.c_int * 3)()
    for T in (1, 3, 20, 31, 33, 50, 64, 100, 128, 200, 256, 300, 611, 1025, 2048, 8000):
        for pairs in (74, 66, 5, 1):
            assert lib.moe_test_ffn_deal(T, h, f, pairs, 0, items, most, deal) == 0
            total, seen = deal[0], []
            for pair in range(min(total, pairs)):
                assert lib.moe_test_ffn_deal(T, h, f, pairs, pair, items, most, deal) == 0
                n, ahead = deal[1], deal[2]
                mine = list(items[:n])
                assert n <= most and ahead == (mine[0] if mine else -1), (T, pairs, pair, mine, ahead)
                seen += mine
            assert sorted(seen) == list(range(total)), (T, pairs)
    assert lib.moe_test_ffn_deal(1, 8, 8, 74, 4, items, most, deal) == -1  # four items: the launch has four pairs
