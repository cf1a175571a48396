"""Every output buffer that mem_rmsnorm is given is written, or refused."""
import pytest
import torch

import paper_2412_09764_amd as pk

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("quantize", [False, True])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("want_sum", [False, True])
def test_sum_out(gpu_lib, dt, quantize, residual, want_sum):
    x = torch.randn((9, 72), generator=torch.Generator().manual_seed(1)).to(dt).cuda()
    r = (x * 2).flip(0).contiguous() if residual else None
    into = torch.full_like(x, 7.0)
    y, h, s = pk.mem_rmsnorm(x, None, r, quantize=quantize, sum_out=into, want_sum=want_sum)
    assert h is into and torch.equal(into, x if r is None else (x.float() + r.float()).to(dt))
    y2, h2, s2 = pk.mem_rmsnorm(x, None, r, quantize=quantize, want_sum=want_sum)
    assert torch.equal(y.float(), y2.float()) and (h2 is None) == (not residual or not want_sum)
    assert (s is None and s2 is None) if not quantize else torch.equal(s, s2)
    x2 = x.clone()
    assert pk.mem_rmsnorm(x2, None, r, quantize=quantize, sum_out=x2)[1] is x2 and torch.equal(x2, into)


def test_scale_out_without_codes_is_refused(gpu_lib):
    x = torch.ones((9, 72), device="cuda")
    with pytest.raises(ValueError):
        pk.mem_rmsnorm(x, scale_out=torch.zeros(9, device="cuda"))
