"""Attention over several thousand tokens: many rounds per block, every barrier's phase used many times."""
import pytest
import torch

from test_gpu_attention import BF, F32, check, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("nq,nk,causal,window", [(5000, 5000, True, 0), (4097, 6001, False, 0), (6000, 6000, True, 1000), (1, 9000, True, 0),
                                                 (130, 8191, True, 500), (5000, 300, True, 0)])
@pytest.mark.parametrize("dtype,d", [(BF, 64), (BF, 128), (F32, 64)])
def test_long(dtype, d, nq, nk, causal, window):
    check(*make(1, nq, nk, 2, 1, d, dtype), causal=causal, window=window)


@pytest.mark.parametrize("d", [64, 128])
def test_long_and_short_documents_in_one_row(d):
    lens = [3, 4000, 1, 700, 128, 2100, 40]
    off = torch.tensor([0] + torch.tensor(lens).cumsum(0).tolist(), dtype=torch.int32, device="cuda")
    q, k, v, do = (t[0] for t in make(1, sum(lens), sum(lens), 2, 1, d, BF))
    check(q, k, v, do, q_offsets=off, k_offsets=off)
