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
