"""Norm rows of every number of lanes and passes: the shapes that test_gpu_norm does not reach, held to the same forms."""

import pytest

import test_gpu_norm as N

pytestmark = pytest.mark.gpu

# 64 lanes with two, three and four passes (more than 1024 rows), 256 with two and with three for few rows and many, 1024 with
# one (up to 512 rows) and three
SHAPES = [(1030, 1000), (1025, 1531), (1100, 2047), (40, 3001), (600, 5001), (5, 5000), (512, 8190), (2, 20000)]


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_lanes(rows, cols, dt):
    N.test_values(rows, cols, dt, "same")
    N.test_codes(rows, cols, dt, True)
    N.test_codes(rows, cols, dt, False)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", [(130, 2049), (1200, 3001), (3, 4096), (40, 5001), (9, 8193), (600, 16384)])
def test_gradient_lanes(rows, cols, dt):
    N.test_gradients(rows, cols, dt)
