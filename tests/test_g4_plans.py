"""The sizes that tests/test_gpu_g4_tiles.py runs take the kernels that they are there for, and together all of them: a change of
the plan's constants must not leave a kernel without a test."""
import pytest

import g4_reference as ref
import g4_shapes


@pytest.fixture(scope="module")
def qnn():
    from paper_2106_09886_b200 import build
    build.build()
    from paper_2106_09886_b200 import qnn as q
    return q


@pytest.mark.parametrize("product,dtype,rows,experts,n,k,tile,split", g4_shapes.EVERY)
def test_shape_takes_its_tile(qnn, product, dtype, rows, experts, n, k, tile, split):
    got = qnn.g4_plan(product, ref.torch_type(dtype), rows, experts, n, k)
    assert got[0] == tile and (got[1] > 1) == split


def test_every_kernel_has_a_shape():
    have = {(product, dtype, tile, split) for product, dtype, *_, tile, split in g4_shapes.EVERY}
    for dtype in ref.TYPES:
        tiles = (32, 64) if dtype == "fp32" else (32, 64, 128, 256)
        assert ("experts", dtype, 0, False) in have
        for product in ("experts", "data"):
            for tile in tiles:
                assert {(product, dtype, tile, False), (product, dtype, tile, True)} <= have
        assert {("weights", dtype, 128, False), ("weights", dtype, 128, True), ("weights", dtype, 256, False)} <= have


def test_plan_refusals(qnn):
    import ctypes
    f = qnn.lib.qnn_g4_plan
    a, b = ctypes.c_int(), ctypes.c_int()
    ok = (0, 0, 1, 10, 2, 64, 64, ctypes.byref(a), ctypes.byref(b))
    assert f(*ok) == qnn.OK
    for at, bad in ((0, 3), (0, -1), (1, 1), (2, 3), (3, 0), (3, -1), (4, 0), (4, 4097), (5, 0), (6, 0), (7, None), (8, None)):
        assert f(*(bad if i == at else v for i, v in enumerate(ok))) == qnn.E_ARG, (at, bad)
    assert f(*(2 ** 31 if i == 3 else v for i, v in enumerate(ok))) == qnn.E_RANGE
    assert qnn.g4_plan("matvec", ref.torch_type("bf16"), 8, 1, 64, 64) == (0, 1)
