"""Which launch copies an eviction's rows (host arithmetic, no GPU): the faster one where both were measured."""
import ctypes

import pytest

from paper_2604_09244_amd import binding as mv

# heads, rows that stay, us with workgroups that copy their rows themselves, with a second launch
OTHER = [(32, 64, 6.6, 7.6), (32, 1344, 21.6, 16.8), (32, 4096, 58.0, 36.8), (64, 1344, 23.4, 19.2), (192, 1344, 28.9, 30.8),
         (192, 4096, 85.5, 78.7), (192, 8192, 167.8, 152.8), (256, 1344, 32.7, 35.6), (256, 8192, 199.2, 188.1),
         (384, 2048, 73.5, 68.7), (384, 4096, 155.3, 135.0), (512, 1344, 57.2, 60.2), (512, 8192, 390.6, 375.8)]
IN_PLACE = [(32, 64, 6.9, 7.7), (32, 512, 11.2, 12.0), (32, 8192, 61.3, 50.8), (64, 2048, 21.6, 20.7), (64, 4096, 35.1, 32.2),
            (64, 8192, 61.7, 53.2), (128, 1344, 17.9, 18.3), (128, 4096, 35.4, 34.0), (128, 8192, 68.0, 60.3), (192, 1344, 18.1, 19.3),
            (192, 2688, 27.0, 27.8), (256, 1344, 18.2, 19.8), (256, 4096, 35.9, 39.5), (512, 1344, 22.1, 25.8)]


@pytest.mark.parametrize("in_place,cases", [(False, OTHER), (True, IN_PLACE)])
def test_the_faster_launch(in_place, cases):
    moves = getattr(mv.load(), "_ZN4mvla17cache_evict_movesEiib")
    moves.argtypes, moves.restype = [ctypes.c_int, ctypes.c_int, ctypes.c_bool], ctypes.c_bool
    for heads, rows, itself, second in cases:
        assert moves(heads, rows, in_place) == (itself < second), (heads, rows)
