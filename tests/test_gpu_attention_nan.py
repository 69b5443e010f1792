"""A NaN in a token that counts shows in every result that the formula makes of it, at every place in a tile."""
import pytest
import torch

from test_gpu_attention import BF, F32, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,d", [(BF, 64), (BF, 128), (BF, 136), (F32, 64)])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("place", [0, 1, 2, 3, 4, 5, 6, 7, 58, 67, 126])
def test_a_query_of_nan_reaches_every_gradient_it_takes_part_in(dtype, d, causal, place):
    from paper_2609_21594_b200 import functional as F

    q, k, v, do = make(1, 512, 512, 2, 1, d, dtype)
    i = 256 + place
    q = q.clone()
    q[0, i, 1] = float("nan")
    o, lse = F.attention_forward(q, k, v, causal)
    dq, dk, dv = F.attention_backward(do, q, k, v, o, lse, causal)
    seen = i + 1 if causal else 512
    assert o[0, i, 1].isnan().all() and lse[0, 1, i].isnan() and dq[0, i, 1].isnan().all()
    assert dk[0, :seen].isnan().all() and dv[0, :seen].isnan().all()
    assert not o[0, :, 0].isnan().any() and not dq[0, :, 0].isnan().any()


@pytest.mark.parametrize("dtype,d", [(BF, 64), (BF, 128), (F32, 64)])
@pytest.mark.parametrize("place", [2, 3, 5, 66])
def test_a_key_of_nan_reaches_every_query_that_sees_it(dtype, d, place):
    from paper_2609_21594_b200 import functional as F

    q, k, v, do = make(1, 512, 512, 2, 1, d, dtype)
    k = k.clone()
    k[0, 128 + place] = float("nan")
    o, lse = F.attention_forward(q, k, v)
    dq, dk, dv = F.attention_backward(do, q, k, v, o, lse)
    assert o[0, 128 + place:].isnan().all() and dq[0, 128 + place:].isnan().all()
    assert dv[0].isnan().all() and dk[0].isnan().all()           # every key is seen by a query after it, whose probabilities are NaN
