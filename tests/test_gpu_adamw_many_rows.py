"""More touched rows than one launch holds (2^24 - 1 workgroups of 32 rows): the rows behind
that place, and one whose gradients lie on both sides of it, are stepped as in a short list."""
import pytest
import torch

import paper_2412_09764_amd as pk

pytestmark = pytest.mark.gpu


def test_rows_past_one_launch(gpu_lib):
    edge, N, D = (1 << 29) - 32, 64, 8
    for U, first in ((edge + 40, edge - 2), (edge + 132, edge + 92)):
        torch.cuda.empty_cache()
        rows = torch.full((U,), -1, dtype=torch.int64, device="cuda")  # passed over
        grads = torch.zeros((U, D), device="cuda")
        live = [first, first + 1, first + 2, first + 3]
        rows[live[0]:live[3]] = 9   # several gradients of one row
        rows[live[3]:] = 40
        short = torch.randn((4, D), generator=torch.Generator().manual_seed(U % 97)).cuda()
        grads[live] = short
        p = torch.randn((N, D), generator=torch.Generator().manual_seed(2)).cuda()
        a, b = p.clone(), p.clone()
        ma, va, _, _ = pk.mem_adamw_state(a)
        mb, vb, _, _ = pk.mem_adamw_state(b)
        pk.mem_adamw_rows(a, rows, grads, ma, va, lr=1e-2, step=3)
        pk.mem_adamw_rows(b, torch.tensor([9, 9, 9, 40], device="cuda"), short, mb, vb, lr=1e-2, step=3)
        for x, y in ((a, b), (ma, mb), (va, vb)):
            assert torch.equal(x, y), U
        assert not torch.equal(a[9], p[9]) and not torch.equal(a[40], p[40])
        del rows, grads
