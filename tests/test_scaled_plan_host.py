"""Host checks of the plans of the 8-bit products with block scales and of their gradients: which kernels the GPU tests of these operators reach, and where
the plans draw their lines (sizes at which both sides were timed)."""
import pytest

from tests import scaled_plan as S
from tests import test_gpu_scaled as T
from tests import test_gpu_scaled_large as L
from tests import test_gpu_scaled_programs as P


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    return S.load(tmp_path_factory.mktemp("scaled_plan"))


def test_shapes_of_the_large_tile_tests_have_large_tiles(lib):
    for shape in L.LARGE + [(2064, 4112, 400), (2304, 4096, 640), (2064, 4128, 400)]:
        assert S.product(lib, *shape, workspace=False) == "256x256", shape


def test_shapes_of_the_few_row_tests_are_one_kernel(lib):
    for shape in L.FEW + [(1, 6144, 1024), (9, 528, 400), (30, 4224, 528)]:
        for ws in (False, True):
            assert S.product(lib, *shape, workspace=ws, narrow=True) == "few", shape


def test_plain_and_8_bit_shapes_without_a_workspace_have_half_tiles(lib):
    for shape in T.SHAPES + T.Q8_SHAPES:
        assert S.product(lib, *shape, workspace=False) == "128x256", shape


# divided shapes among those of the plain tests: 32, 64 and 128 rows
@pytest.mark.parametrize("shape,plan", [((1, 272, 4096), ("32x128", 16)), ((33, 528, 1040), ("64x128", 9)), ((64, 1024, 2048), ("64x128", 8)),
                                        ((65, 272, 784), ("128x128", 7)), ((257, 512, 1168), ("128x128", 5)), ((300, 784, 2064), ("128x128", 6)),
                                        ((1, 512, 4096), ("32x128", 16))])
def test_shapes_that_are_divided(lib, shape, plan):
    assert shape in T.SHAPES + T.Q8_SHAPES
    assert S.product(lib, *shape, workspace=True) == plan


# where the tests of every program take partials
@pytest.mark.parametrize("shape,tile", zip(P.DIVIDED, ["32x128", "64x128", "128x128", "128x128"]))
def test_divided_shapes_of_the_program_tests(lib, shape, tile):
    plan = S.product(lib, *shape, workspace=True)
    assert plan[0] == tile and plan[1] > 1 and shape[0] % 4 and shape[1] % 256


def test_undivided_shapes_of_the_program_tests(lib):
    for shapes, tile in ((P.HALF, "128x256"), (P.LARGE, "256x256")):
        for shape in shapes:
            assert S.product(lib, *shape, workspace=False) == tile
    assert any(M % 256 == N % 256 == K % 128 == 0 for M, N, K in P.LARGE) and any(M % 256 and N % 256 and K % 128 for M, N, K in P.LARGE)


# gradients of the GPU tests: undivided 128 x 128, divided, 256 x 256
@pytest.mark.parametrize("shape,plan", [((16, 16, 1), (128, 1)), ((400, 144, 1000), (128, 4)), ((2048, 4096, 70), (128, 1)), ((2064, 4112, 333), (256, 1)),
                                        ((4112, 2064, 1000), (256, 1)), ((4096, 4096, 320), (256, 1)), ((4096, 4096, 257), (256, 1)), ((4096, 4104, 320), (256, 1)),
                                        ((16384, 16, 140016), (128, 4)), ((16384, 528, 140016), (256, 1))])
def test_tiles_of_gradients(lib, shape, plan):
    assert S.gradient(lib, *shape, workspace=True) == plan and S.gradient(lib, *shape, workspace=False) == (plan[0], 1)


# without a workspace (microseconds: 128 x 256 tiles, 256 x 256 tiles)
@pytest.mark.parametrize("shape,tile", [((1000, 4096, 14336), "128x256"),          # 78, 126
                                        ((1039, 14336, 4096), "128x256"),          # 66, 95
                                        ((4608, 4608, 4096), "128x256"),           # 92, 95
                                        ((2500, 4608, 2048), "256x256"),           # 35.7, 30.8
                                        ((2048, 8192, 4096), "256x256"),           # 66, 56
                                        ((8192, 16384, 2048), "256x256")])         # 300, 254
def test_tiles_where_they_are_faster(lib, shape, tile):
    assert S.product(lib, *shape, workspace=False) == tile


# with one (microseconds: divided, one kernel)
@pytest.mark.parametrize("shape,plan", [((215, 4224, 10416), ("128x128", 3)),      # 26.4 (4 ranges: 38.3)
                                        ((33, 11264, 2048), ("64x128", 2)),        # 10.9 (3 ranges: 12.9)
                                        ((1000, 2048, 5632), ("128x128", 2)),      # 24.8, 33.9
                                        ((300, 2048, 2048), ("128x128", 4)),       # 14.3, 16.1
                                        ((96, 2048, 1024), ("128x128", 4)),        # 8.7, 11.4
                                        ((614, 5600, 1584), "128x256"),            # 23.0, 18.7
                                        ((300, 2048, 256), "128x256")])            # 7.1, 7.4: level, a launch less
def test_ranges_where_they_are_faster(lib, shape, plan):
    assert S.product(lib, *shape, workspace=True) == plan


# one kernel for few rows where it was the faster, partials where they were
@pytest.mark.parametrize("shape,few", [((1, 6144, 4096), True), ((8, 6144, 4096), True), ((16, 6144, 4096), True), ((32, 6144, 4096), False),
                                       ((1, 4096, 14336), True), ((8, 4096, 14336), True), ((24, 4096, 14336), False), ((1, 16384, 2048), True),
                                       ((24, 4096, 4096), True), ((1, 28672, 4096), False)])
def test_few_rows_where_one_kernel_is_faster(lib, shape, few):
    assert (S.product(lib, *shape, workspace=True, narrow=True) == "few") == few


# M, N, tokens (microseconds: 256 x 256 tiles, 128 x 128 tiles)
@pytest.mark.parametrize("shape,tile", [((2048, 4096, 320), 128),            # 22.9, 18.7: 512 tiles of 128 x 128, one round
                                        ((2048, 4096, 1000), 128),           # 39.6, 30.6
                                        ((2048, 4096, 4096), 128),           # 114, 86
                                        ((1024, 8192, 320), 128),            # 22.9, 18.6
                                        ((256, 32768, 4096), 128),           # 114, 86
                                        ((256, 34816, 1000), 256),           # 40.1, 45.0: 544
                                        ((2304, 4096, 320), 256),            # 23.8, 24.3
                                        ((2304, 4096, 4096), 256),           # 114, 137
                                        ((5632, 2048, 1000), 256),           # 43.6, 48.8
                                        ((4096, 4096, 4096), 256),           # 127, 157
                                        ((2048, 16384, 8192), 256),          # 470, 608
                                        ((4096, 14336, 256), 128),           # 126, 115
                                        ((4096, 14336, 64), 128),            # 107, 102
                                        ((2048, 2048, 2048), 128)])          # 62, 38.5
def test_gradient_tiles_where_they_are_faster(lib, shape, tile):
    assert S.gradient(lib, *shape, workspace=True) == S.gradient(lib, *shape, workspace=False) == (tile, 1)


def test_gradient_of_few_tiles_in_ranges(lib):
    assert S.gradient(lib, 512, 1024, 8192, workspace=True) == (128, 16)            # 26.9, undivided 116
    assert S.gradient(lib, 400, 144, 1000, workspace=True) == (128, 4)              # 10.1, 18.4
    for M, N, K in ((16, 32528, 1000), (16, 32768, 1000), (128, 65536, 1000)):      # one row of tiles: no more than a round of them
        tile, ranges = S.gradient(lib, M, N, K, workspace=True)
        assert tile == 128 and -(-M // 128) * -(-N // 128) * ranges <= 512
