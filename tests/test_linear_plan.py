"""Which kernels the projections' rules choose, on the host."""
import shutil

import pytest

from tests.linear_plan import TILES, Plan
from tests.test_gpu_linear_tiles import BACKWARD, FORWARD


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    if not shutil.which("g++"):
        pytest.skip("no g++")
    return Plan(str(tmp_path_factory.mktemp("plan")))


def test_every_kernel_is_reached(plan):
    """The sizes that the GPU tests run take each kernel at least once: a changed rule may
    not drop one unseen."""
    types = ("f32", "bf16")
    reached = {("forward", dt, "few rows" if T <= 8 else plan.product(dt, T, N)) for T, N, K in FORWARD
               for dt in (*types, "e4m3")}
    reached |= {("dx", dt, plan.product(dt, T, K)) for T, N, K in BACKWARD for dt in types}
    for T, N, K in BACKWARD:
        for dt in types:
            tile, splits = plan.grad(dt, T, N, K)
            reached.add(("grad_w", dt, tile, splits > 1))
    wanted = {("forward", dt, t) for dt in (*types, "e4m3") for t in ("few rows", *TILES)}
    wanted |= {("dx", dt, t) for dt in types for t in TILES}
    wanted |= {("grad_w", dt, t, split) for dt in types for t in TILES if t != "128" for split in (False, True)}
    assert not wanted - reached, sorted(wanted - reached)
    assert not reached - wanted, sorted(reached - wanted)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "e4m3"])
def test_few_rows_of_wide_products(plan, dtype):
    """No 256-wide tiles for up to 128 rows, and 128-wide ones for up to 64 only where a wide
    product has more than 192 of them."""
    for M in (9, 16, 33, 64, 65, 100, 128, 129, 200):
        for N in (8, 2048, 16384, 24576, 25608, 51200, 131072, 1 << 20):
            tile = plan.product(dtype, M, N)
            assert tile != "256" or M > 128, (M, N)
            assert not tile.startswith("128") or M > 64 or -(-N // 128) > 192, (M, N)
