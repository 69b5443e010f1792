"""Products that keep the device busy for a long time: a bounded wait is for what does not come, not for what takes long."""
import pytest
import torch

import feed_forward_reference as ref

pytestmark = pytest.mark.gpu


def test_a_launch_of_half_a_second_reports_no_expired_wait():
    """57344 tokens of 57344 x 57344: 0.45 s in the gated product alone, 40 GB.  Some rows of the result against 64 bits."""
    from paper_2609_21594_b200 import functional as F

    n = 57344
    if torch.cuda.mem_get_info()[0] < 50e9:
        pytest.skip("50 GB of free memory are needed")
    F.synchronize_and_check()
    g = torch.Generator(device="cuda").manual_seed(0)
    x, *w = (torch.empty((n, n), dtype=torch.bfloat16, device="cuda").normal_(0, s, generator=g) for s in (1, n ** -0.5, n ** -0.5, n ** -0.5))
    y, _ = F.feed_forward_forward(x, *w, "silu", "none")
    torch.cuda.synchronize()
    expired = F.context().muon_last_device_status()
    F.context().muon_clear_device_status()                   # the word is every later call's, too
    assert expired == 0
    rows = torch.tensor([0, 1, 255, 256, 31000, n - 1], device="cuda")
    cut = lambda a, b: torch.cat([a @ b[i:i + 4096].double().T for i in range(0, n, 4096)], 1)  # noqa: E731
    xr = x[rows].double()
    h = (ref.act(cut(xr, w[0]), "silu") * cut(xr, w[1])).bfloat16().double()
    value = cut(h, w[2])
    # the result's rounding and what fp32 sums turn in those of h, beside which a tile that was left out stands out
    assert float((y[rows].double() - value).norm() / value.norm()) < 2 * ref.half(torch.bfloat16)
    del x, w, y
    torch.cuda.empty_cache()
