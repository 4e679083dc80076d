"""The corners of the 8-bit paged cache: rows and masses at the ends of their ranges, calls as large as the header allows, and what the
sums' logarithms and the weights lose."""
import math
import sys

import pytest

pytestmark = pytest.mark.gpu

D = 128
U32 = 2.0 ** -24


def say(*a):
    print(*a, file=sys.stderr, flush=True)


@pytest.fixture(scope="module")
def vr():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a visible MI355X")
    import paper_2607_15498_amd as vr
    vr.library()
    return vr


@pytest.fixture(scope="module")
def R():
    import paged8_ref
    return paged8_ref


# ---- eviction: rows of zeros beside large ones -----------------------------------------------------

@pytest.mark.parametrize("big", [3e8, 2.0 ** 20 * 448, 2.0 ** 60, 2.0 ** 127])
@pytest.mark.parametrize("small", [0.0, 2.0 ** -118, 2.0 ** -100, 1.0])
def test_evict_zero_rows_of_large_blocks(vr, R, big, small):
    """Rows of zeros (with NaN among them, too) whose block has a large power of two, alone, beside rows of other blocks and beside the
    large row: zeros stay zeros."""
    import torch
    from test_gpu_paged8 import check_evict
    n, keep = 96, 33
    for stay in ([0, 1, 2, 3], [0, 1, 6, 40, 41], [0, 6], [0, 5, 6, 70], list(range(32)) + [40], list(range(6, 32)) + [33, 70]):
        pool = R.Pool8([n], 2, 32, 1, spare=2, fill=False, junk=0.0)
        for x in "kv":
            rows = torch.zeros((n, 2, D))
            rows[5, 0, 7] = big
            rows[6, 0, 9], rows[31, 0, 0] = math.nan, -0.0
            rows[32:64, 0, 3] = small
            rows[64:, 0] = torch.randn((32, D), generator=torch.Generator().manual_seed(3)) * small
            rows[:, 1] = torch.randn((n, D), generator=torch.Generator().manual_seed(2))
            pool.append_rows(0, 0, rows, x)
        mass = torch.zeros((1, 2, n))
        mass[0, :, stay] = 1.0
        check_evict(vr, R, [n], len(stay) if len(stay) < keep else keep, 2, 32, pool=pool, mass=mass)
