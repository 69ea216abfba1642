"""Which kernel a microscaled product's size gets, read from the built library (no GPU): the sizes below reach every one that there is, with k in one part and in more,
and with one plane of activations (16 bits) and three (32 bits).  test_gpu_mx4_epilogue_kernels.py runs them."""
import ctypes as C

import pytest

from paper_2603_02599_amd import binding as sun

FEW, STREAM, TILE = 0, 1, 2
# (columns of all matrices together, k, rows), and what each of one and three planes gets: (kind, row tiles of a wave, columns of a workgroup, whether k is split).  Rows and columns leave a
# remainder everywhere; columns and halves of them are multiples of four in some and not in others.
SIZES = [
    ((130, 96, 5), (FEW, 1, 16, False), (FEW, 1, 16, False)), ((130, 1056, 11), (FEW, 1, 16, False), (FEW, 1, 32, False)),
    ((4504, 160, 7), (FEW, 1, 32, False), (FEW, 1, 32, False)), ((4502, 96, 13), (FEW, 1, 32, False), (FEW, 1, 64, False)),
    ((8204, 160, 3), (FEW, 1, 64, False), (FEW, 1, 64, False)), ((8202, 96, 15), (FEW, 1, 64, False), (FEW, 1, 64, False)),
    ((136, 160, 17), (STREAM, 2, 64, False), (STREAM, 2, 64, False)), ((130, 3104, 31), (STREAM, 2, 64, True), (STREAM, 2, 64, True)),
    ((136, 160, 63), (STREAM, 4, 64, False), (STREAM, 4, 64, False)), ((130, 2080, 33), (STREAM, 4, 64, True), (STREAM, 4, 64, True)),
    ((136, 160, 101), (STREAM, 8, 64, False), (STREAM, 8, 64, False)), ((130, 2080, 65), (STREAM, 8, 64, True), (STREAM, 8, 64, True)),
    ((16504, 160, 17), (STREAM, 2, 128, False), (STREAM, 2, 128, False)), ((2050, 4096, 17), (STREAM, 2, 128, True), (STREAM, 2, 128, True)),
    ((16504, 160, 40), (STREAM, 4, 128, False), (STREAM, 4, 128, False)), ((2050, 4096, 40), (STREAM, 4, 128, True), (STREAM, 4, 128, True)),
    ((16504, 160, 101), (STREAM, 8, 128, False), (STREAM, 8, 128, False)), ((2050, 4096, 101), (STREAM, 8, 128, True), (STREAM, 8, 128, True)),
    ((136, 160, 129), (TILE, 4, 128, False), (TILE, 4, 128, False)), ((130, 1376, 131), (TILE, 4, 128, True), (TILE, 4, 128, True)),
    ((16504, 160, 385), (TILE, 5, 256, False), (TILE, 5, 256, False)), ((2050, 4096, 385), (TILE, 5, 256, True), (TILE, 5, 256, True)),
    ((10008, 160, 1001), (TILE, 6, 256, False), (TILE, 6, 256, False)), ((1030, 4096, 1001), None, (TILE, 6, 256, True)), ((1302, 4096, 900), (TILE, 6, 256, True), None),
    ((16504, 160, 599), (TILE, 7, 256, False), (TILE, 7, 256, False)), ((3002, 4096, 385), (TILE, 7, 256, True), None), ((1302, 4096, 1001), None, (TILE, 7, 256, True)),
    ((16504, 160, 701), (TILE, 8, 256, False), (TILE, 8, 256, False)), ((16504, 3104, 225), (TILE, 8, 256, True), None), ((1602, 4096, 900), None, (TILE, 8, 256, True)),
]
KERNELS = {(FEW, 1, cols, False) for cols in (16, 32, 64)} | {(STREAM, rt, cols, split) for rt in (2, 4, 8) for cols in (64, 128) for split in (False, True)} | {
    (TILE, rt, 128 if rt == 4 else 256, split) for rt in (4, 5, 6, 7, 8) for split in (False, True)}


class Plan(C.Structure):
    _fields_ = [(n, C.c_int) for n in ("kind", "rt", "cols", "splits")]


@pytest.fixture(scope="module")
def plan():
    f = sun.lib()._ZN3sun8mx4_planEiiii   # Mx4Plan sun::mx4_plan(int N, int K, int rows, int planes)
    f.restype, f.argtypes = Plan, [C.c_int] * 4

    def of(size, planes):
        p = f(*size, planes)
        return p.kind, p.rt, p.cols, p.splits > 1
    return of


@pytest.mark.parametrize("size, one, three", SIZES)
def test_a_size_gets_the_kernel_that_it_is_here_for(plan, size, one, three):
    for planes, want in ((1, one), (3, three)):
        if want is not None:
            assert plan(size, planes) == want, planes


def test_the_sizes_reach_every_kernel(plan):
    assert KERNELS == {one for _, one, _ in SIZES if one} == {three for _, _, three in SIZES if three}
    for n in (17, 130, 1030, 2050, 3002, 4096, 5120, 8250, 14336, 16502, 28672, 200000):   # and there is no other
        for k in (32, 352, 2080, 4096, 14336):
            for rows in (1, 9, 16, 17, 32, 33, 64, 65, 128, 129, 160, 161, 192, 200, 224, 256, 300, 400, 513, 1000, 3000):
                for planes in (1, 3):
                    assert plan((n, k, rows), planes) in KERNELS, (n, k, rows, planes)
