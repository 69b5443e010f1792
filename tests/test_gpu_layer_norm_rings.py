"""Layer norm where a row group comes back to its places in shared memory many times, and where two blocks share a row."""
import pytest
import torch

from test_gpu_layer_norm import check_backward, check_forward, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,cols", [(1, 8200), (2, 16384), (5, 12288), (333, 9001)])
def test_rows_cut_between_two_blocks_keep_their_sums(dtype, rows, cols):
    """The blocks of a pair start at their own times, most of all when others hold the SMs: the same bits on every launch."""
    from paper_2609_21594_b200 import functional as F

    x, w, b, dy = make(rows, cols, dtype, torch.float32)
    mean, rstd = check_forward(x, w, b, 1e-5, True)
    want = check_backward(dy, x, w, mean, rstd)
    wide = make(600, 16384, torch.bfloat16, torch.float32, seed=1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(40):
        with torch.cuda.stream(side):
            F.layer_norm_forward(*wide[:3])
        got = F.layer_norm_backward(dy, x, w, mean, rstd)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    torch.cuda.current_stream().wait_stream(side)


@pytest.mark.parametrize("center", [True, False])
@pytest.mark.parametrize("rows,cols", [(5000, 40), (5000, 256), (3000, 512), (2500, 1024), (1300, 4096), (1000, 8192), (700, 12288), (700, 16384), (900, 1001)])
def test_many_fp32_rows_per_group(rows, cols, center):
    """fp32 rows by pieces: two places ahead forward (one above 8192 columns), three backward, each used several times."""
    x, w, b, dy = make(rows, cols, torch.float32, torch.float32)
    mean, rstd = check_forward(x, w, b, 1e-5, center)
    check_backward(dy, x, w, mean, rstd)
