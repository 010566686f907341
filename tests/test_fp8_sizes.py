"""The sizes that products in 8 bits are tested at take every way that a product may take, whatever becomes of the model that chooses: said by the host code, without a GPU."""
import ctypes as C
import os

import pytest

from test_gpu_lowbit_fp8_sums import SIZES

BF16, FP16, FP32 = 0, 1, 2
FEW, INSIDE = -1, -2
# (tile or kernel, with splits of the columns, waves, tiles of sixteen tokens)
INSIDE_WAYS = {(INSIDE, False, waves, 1) for waves in (2, 4, 8)}
FEW_WAYS = {(FEW, False, waves, tiles) for waves, tiles in ((2, 1), (4, 1), (2, 2), (4, 2), (2, 4))}
TILES = {(shape, splits, 0, 0) for shape in (3, 4, 5, 6) for splits in (False, True)}
LARGE = {(shape, False, 0, 0) for shape in (0, 1, 2)}


@pytest.fixture(scope="module")
def way():
    from paper_2604_03298_amd import build
    if not os.path.exists(build.TEST_LIB):
        build.build()
    plan = C.CDLL(build.TEST_LIB).enec_test_fp8_plan
    plan.restype, plan.argtypes = None, [C.c_size_t, C.c_size_t, C.c_size_t, C.c_int, C.c_int, C.POINTER(C.c_int32)]

    def way(m, n, k, dtype, linear):
        out = (C.c_int32 * 4)()
        plan(m, n, k, dtype, linear, out)
        return out[0], out[1] > 1, out[2], out[3]
    return way


@pytest.mark.parametrize("dtype, linear, ways", [(BF16, 0, FEW_WAYS | TILES | LARGE), (BF16, 1, INSIDE_WAYS | TILES | LARGE), (FP16, 0, FEW_WAYS | TILES), (FP16, 1, INSIDE_WAYS | TILES),
                                                 (FP32, 0, FEW_WAYS | TILES)])
def test_the_tested_sizes_take_every_way(way, dtype, linear, ways):
    taken = {way(m, n, k, dtype, linear) for m, n, k in SIZES}
    assert ways <= taken, sorted(ways - taken)
    assert taken <= ways | FEW_WAYS


@pytest.mark.parametrize("k", [2049, 2560, 3328, 4096])
def test_rows_of_weights_do_not_change_the_waves_of_long_rows(way, k):
    """One rule for all of them: with weights from memory four waves are better, or as good, over the whole range."""
    assert {way(1, n, k, BF16, 1) for n in (16, 300, 4096, 8192, 8193, 11008, 12288, 12289, 32003, 70000)} == {(INSIDE, False, 4, 1)}
