"""CPU: which kernel a product of 8-bit operands takes (csrc/linear8_plan.hpp, compiled on the host)."""
import ctypes
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2201_13195_amd", "csrc")
FEW_16x16, FEW_16x32, FEW_32x32, FEW_64x32, MANY_16x64, MANY_32x32, MANY_64x32, TILE_64x128, TILE_128_SPLIT, TILE_128, TILE_256 = range(11)
UNITS = 256

# (n, d_in, d_out) of each kernel, bf16 and fp32 results; tests/test_gpu_linear8.py runs them.
KERNELS = [
    ((5, 200, 70), FEW_16x16, FEW_16x16), ((256, 512, 256), FEW_16x16, FEW_16x16),
    ((16, 1000, 5000), FEW_16x32, FEW_16x32), ((130, 777, 800), FEW_16x32, FEW_16x32),
    ((60, 300, 3001), FEW_32x32, FEW_32x32), ((500, 900, 510), FEW_32x32, FEW_32x32),
    ((333, 1000, 1111), MANY_32x32, MANY_32x32), ((333, 1030, 1111), FEW_64x32, FEW_64x32), ((128, 2048, 4000), FEW_64x32, FEW_64x32),
    ((1, 520, 9001), MANY_16x64, MANY_16x64), ((16, 136, 20000), MANY_16x64, MANY_16x64),
    ((20, 520, 9001), MANY_32x32, MANY_32x32), ((32, 131, 17000), MANY_32x32, MANY_32x32),
    ((600, 400, 1200), MANY_64x32, MANY_64x32), ((50, 777, 17000), MANY_64x32, MANY_64x32), ((256, 2100, 4001), MANY_64x32, MANY_64x32), ((1100, 2050, 1030), TILE_64x128, TILE_64x128),
    ((500, 777, 3000), TILE_64x128, TILE_64x128),     # seven blocks: the second group has none in the last step
    ((260, 1160, 4090), TILE_64x128, TILE_64x128), ((100, 1111, 9000), TILE_64x128, TILE_64x128),
    ((900, 2600, 4000), TILE_128_SPLIT, TILE_128_SPLIT), ((2000, 2440, 2040), TILE_128_SPLIT, TILE_128_SPLIT),
    ((1500, 2513, 2500), TILE_128_SPLIT, TILE_128_SPLIT), ((700, 600, 4000), TILE_128, TILE_128),
    ((2100, 250, 4100), TILE_128, TILE_128),          # more tiles than places, two steps: a work-group has a second tile
    ((2100, 128, 4100), TILE_128, TILE_128),          # one step
    ((4096, 1024, 4096), TILE_256, TILE_128), ((4300, 1000, 4090), TILE_256, TILE_128),      # (the second: two rounds of tiles)
    ((5000, 512, 5000), TILE_256, TILE_128), ((9000, 384, 4104), TILE_256, TILE_128),
]


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    where = tmp_path_factory.mktemp("plan")
    src = where / "plan.cpp"
    src.write_text('#include "linear8_plan.hpp"\nextern "C" int plan(int64_t n, int64_t d_in, int64_t d_out, int64_t x, int64_t w, bool exact) '
                   "{ return rmm::linear8_plan(n, d_in, d_out, x, w, exact); }\n")
    lib = str(where / "plan.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-I" + CSRC,
                    str(src), "-o", lib], check=True)
    f = ctypes.CDLL(lib).plan
    f.restype, f.argtypes = ctypes.c_int, [ctypes.c_int64] * 5 + [ctypes.c_bool]
    return lambda n, d_in, d_out, exact=False, x=None, w=None: f(n, d_in, d_out, x or (d_in + 15) // 16 * 16, w or (d_in + 15) // 16 * 16, exact)


def groups(n, d_out, tokens, outputs):
    return -(-n // tokens) * -(-d_out // outputs)


@pytest.mark.parametrize("shape,bf16,f32", KERNELS)
def test_kernels_by_shape(plan, shape, bf16, f32):
    assert plan(*shape) == bf16 and plan(*shape, exact=True) == f32


def test_every_kernel_is_among_them():
    assert {k for _, k, _ in KERNELS} == set(range(11))


def test_few_outputs_take_the_kernels_without_tiles(plan):
    for n in (1, 2, 15, 16, 17, 31, 33, 64, 65, 100, 128, 200, 333, 512, 1000, 2048):
        for d_in in (100, 1024, 1030, 4096):
            for d_out in (1, 16, 17, 100, 128, 700, 1024, 1111, 2048, 4096, 5000, 8192, 9000, 20000):
                k, short = plan(n, d_in, d_out), d_in <= 1024
                sizes = {FEW_16x16: (16, 16), FEW_16x32: (16, 32), FEW_32x32: (32, 32), FEW_64x32: (64, 32)}
                fit = [j for j in sorted(sizes) if groups(n, d_out, *sizes[j]) <= UNITS]
                two = n > 16 and short and groups(n, d_out, 32, 32) <= 2 * UNITS
                if fit and not (fit[0] == FEW_64x32 and two):
                    assert k == fit[0]                              # the smallest that is one round of work-groups
                elif n <= 16:
                    assert k == MANY_16x64
                elif n <= 32 or two:
                    assert k == MANY_32x32
                else:
                    assert (k == MANY_64x32) == (n <= 64 or groups(n, d_out, 64, 32) <= 2 * UNITS)


def test_groups_that_share_the_contraction_have_a_compute_unit_each(plan):
    for n in (33, 100, 333, 512, 1000, 1024, 2048, 4096):
        for d_out in (100, 1024, 2048, 3000, 4096, 9000, 20000):
            for d_in in (64, 400, 768, 1024, 2500, 4096):
                for exact in (False, True):
                    k = plan(n, d_in, d_out, exact)
                    if k < TILE_64x128:
                        continue
                    half, whole, steps = groups(n, d_out, 64, 128), groups(n, d_out, 128, 128), -(-d_in // 128)
                    assert (k == TILE_64x128) == (half <= UNITS and steps >= (3 if exact else 6))
                    assert (k == TILE_128_SPLIT) == (k != TILE_64x128 and whole <= UNITS and steps >= 20)


def test_large_ones_take_the_large_tile(plan):
    assert plan(16384, 4096, 4096) == plan(16384, 1024, 4096) == plan(16384, 4096, 1024) == TILE_256
    assert plan(8192, 1024, 1024) == plan(4096, 768, 768) == plan(2048, 2048, 2048) == TILE_128
    assert all(plan(20000, d, d, exact=True) == TILE_128 for d in (1000, 4096)) and plan(2100, 1000, 1000, exact=True) == TILE_128


def test_operands_beyond_32_bits_of_a_tile(plan):
    """Rows whose tile does not fit 32-bit offsets, outputs whose tiles do not fit a launch: the kernels with 64-bit addresses."""
    assert plan(5000, 1 << 23, 500) == plan(5000, 500, 500, x=1 << 23) == plan(5000, 500, 500, w=1 << 23) == MANY_32x32
    assert plan((1 << 31) - 1, 16, 500) != TILE_256 and plan((1 << 31) - 1, 1, 511) == MANY_32x32
    for n in (1, 1000, (1 << 31) - 1):
        for d in (1, 1000, (1 << 31) - 1):
            for o in (1, 1000, (1 << 31) - 1):
                if n * d < 1 << 40 and n * o < 1 << 40 and d * o < 1 << 40:
                    assert 0 <= plan(n, d, o) <= TILE_256 and 0 <= plan(n, d, o, exact=True) < TILE_256
